// The backward pass of a 1x1, stride-1 block whose input was kept packed (convbn_tune_bwd_packed), in one kernel:
//     dX = dZ omega' (+ add) (masked by X > 0),      domega' = dZ^T X,      sum dZ
// for the layers and with the products of umma_bwd1x1.cu (WIDE_IN: C_in = 128 or 256, C_out = 64; WIDE_OUT the other way round), with X
// as 8-bit codes and steps (convbn_pack).  Memory: dZ 2 C_out + X (1 + 1/32) C_in + dX and addend 2 C_in each per pixel, all once.
//
// Eight warps restore X on its way into shared memory: a warp requests its 16 pixels of the next tile while it turns those of this one
// into the swizzled 16-bit boxes that the weight-gradient MMAs read (code * step, exact).  The same boxes are the mask of dX: the
// epilogue reads them as matrix fragments beside its accumulator.  Its boxes of the addend arrive by TMA where the results will
// leave from.  Warps: 0 dZ by TMA, 1 MMA issuer and owner of tensor memory, 2-9 epilogue, 10-17 codes to X.
// Measured (launch to launch, inputs cold, bf16): 256 -> 64 at 56 x 56, N = 256 with addend and mask 197-203 us, 0.87 of the copy
// bandwidth on the bytes above (the kernel that reads X itself: 275); 64 -> 256 at N = 32 26.4 us (29.4).
#include "kernels.h"
#include "mma_sync.cuh"
#include "pack8.cuh"
#include "packed_f32.cuh"
#include "sm100_ptx.cuh"

namespace convbn {

using namespace ptx;

namespace {

constexpr int kPbThreads = 576;
constexpr uint32_t kPbBox = 128 * 128;        // [128 pixels][64 channels] of 16 bits
constexpr uint32_t kPbOut = 32 * 128;         // an epilogue warp's box: [32 pixels][64 channels]
// Half values: the accumulators of domega and sum dZ are added to the CTA's partial, which stays in L2, every eight tiles, by additions
// that round (those of the tensor core cut off, and drift: see kExactPixels).  256 -> 64 at 56 x 56, N = 256 204 -> 214 us, 64 -> 128 at
// 100 x 65, N = 240 129 -> 139 (144 in two rounds of CTAs); read back and stored instead 245 and 332, by as many more CTAs 251 and 230.
constexpr uint32_t kPbSegment = 8;

struct PackedBwd {
    long long p;
    int m_tiles;
    const float *vec3;      // saved [s | b' | r]
    int f16;
    const uint8_t *codes, *steps;
    int add, mask;
};

struct PbCtl {
    uint64_t dz_full[2], dz_empty[2], x_full[2], x_empty[2], dx_full[2], dx_empty[2], add_full[8], seg_full, seg_empty, acc_done;
    uint32_t tmem_base;
    int abort_flag;
};

template <int CI, int CO>
struct PbShape {
    static constexpr bool kWideIn = CI >= CO;
    static constexpr int kXBoxes = CI / 64, kDzBoxes = CO / 64;
    static constexpr int kDxBufs = CI <= 128 ? 2 : 1;                    // dX accumulators [128][CI]
    static constexpr int kOutBufs = CI * CO <= 8192 ? 2 : 1;             // boxes of an epilogue warp
    static constexpr int kWide = kWideIn ? CI : CO, kNarrow = kWideIn ? CO : CI;
    static constexpr int kMBlocks = kWide / 128;                         // weight-gradient M blocks
    static constexpr int kDwCol0 = CI * kDxBufs;                         // [kWide][kNarrow] accumulators
    static constexpr int kSumCol0 = kDwCol0 + kMBlocks * kNarrow;
    static constexpr int kSumCols = kWideIn ? CO : 16 * kMBlocks;
    static constexpr size_t kSmem = 1024 + 2 * (size_t)(kXBoxes + kDzBoxes) * kPbBox + (size_t)CI * CO * 2 + 1024 +
                                    8 * (size_t)kOutBufs * kPbOut + sizeof(PbCtl) + 16;
    static_assert(kSumCol0 + kSumCols <= 512, "tensor memory");
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

template <int CI, int CO, bool H>
__global__ void __launch_bounds__(kPbThreads) packed_bwd1x1_kernel(const __grid_constant__ CUtensorMap tm_dz,
                                                                   const __grid_constant__ CUtensorMap tm_dx,
                                                                   const __grid_constant__ CUtensorMap tm_add, const PackedBwd g,
                                                                   const __nv_bfloat16 *__restrict__ w, float *__restrict__ partials,
                                                                   float *__restrict__ bsum, int *err) {
    using S = PbShape<CI, CO>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *x_tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);     // 2 x [CI / 64] boxes
    uint8_t *dz_tiles = x_tiles + 2 * (size_t)S::kXBoxes * kPbBox;                       // 2 x [CO / 64] boxes
    uint8_t *wres = dz_tiles + 2 * (size_t)S::kDzBoxes * kPbBox;     // omega' as [ci / 64][co][64 ci], swizzled
    uint8_t *staging = wres + (size_t)CI * CO * 2;
    uint8_t *ones = staging + 8 * (size_t)S::kOutBufs * kPbOut;      // 8 rows of 64 times 1.0 (read with all strides 0)
    PbCtl *ctl = (PbCtl *)(ones + 1024);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &ctl->abort_flag;
    const int tile_lo = (int)((long long)g.m_tiles * blockIdx.x / gridDim.x);
    const int tile_hi = (int)((long long)g.m_tiles * (blockIdx.x + 1) / gridDim.x);

    if (threadIdx.x == 0) {
        for (int s = 0; s < 2; ++s) {
            mbar_init(&ctl->dz_full[s], 1); mbar_init(&ctl->dz_empty[s], 1);
            mbar_init(&ctl->x_full[s], 8); mbar_init(&ctl->x_empty[s], 1 + (S::kDxBufs == 2 ? 4 : 8));
            mbar_init(&ctl->dx_full[s], 1); mbar_init(&ctl->dx_empty[s], S::kDxBufs == 2 ? 4 : 8);
        }
        for (int s = 0; s < 8; ++s) mbar_init(&ctl->add_full[s], 1);
        mbar_init(&ctl->seg_full, 1); mbar_init(&ctl->seg_empty, 8);
        mbar_init(&ctl->acc_done, 1);
        ctl->abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tm_dz); prefetch_tensormap(&tm_dx);
    }
    if (warp == 1) {
        tmem_alloc(&ctl->tmem_base, 512);
        tmem_relinquish();
    }
    {
        const uint32_t one2 = one_h16(g.f16) * 0x10001u;
        if (threadIdx.x < 64) ((uint4 *)ones)[threadIdx.x] = make_uint4(one2, one2, one2, one2);
        fence_proxy_async_smem();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pdl_wait();
    const uint32_t tmem_base = ctl->tmem_base;
    auto give_up = [&]() { atomicOr(err, ERRW_TIMEOUT); ctl->abort_flag = 1; };

    if (warp == 0) {
        int s = 0, issued = 0;
        uint32_t ph = 1;
        bool ok = true;
        if (elect_one()) {
            for (int t = tile_lo; t < tile_hi; ++t) {
                ok = mbar_wait_bounded(&ctl->dz_empty[s], ph, abort_flag);
                if (!ok) break;
                mbar_arrive_expect_tx(&ctl->dz_full[s], S::kDzBoxes * kPbBox);
                tma_load_3d(dz_tiles + (size_t)s * S::kDzBoxes * kPbBox, &tm_dz, &ctl->dz_full[s], 0, t * 128, 0);
                ++issued;
                if (++s == 2) { s = 0; ph ^= 1u; }
            }
        }
        if (!ok) {
            give_up();
            for (int j = issued > 2 ? issued - 2 : 0; j < issued; ++j)
                mbar_wait_bounded(&ctl->dz_full[j & 1], (uint32_t)(j >> 1) & 1u, nullptr, 200000000ull);
        }
    } else if (warp == 1) {
        named_bar_sync(1, 288);                       // omega' is there (written by warps 2 to 9)
        if (elect_one()) {
            const uint32_t hi = smem_desc_hi_sw128(1024);
            constexpr uint32_t kBox16 = kPbBox >> 4;
            const uint32_t idesc_dx = idesc_h16_f32(128, CI, 0, 1, g.f16);          // A = dZ (K-major), B = omega' (MN-major)
            const uint32_t idesc_dw = idesc_h16_f32(128, S::kNarrow, 1, 1, g.f16);  // both operands MN-major
            const uint32_t idesc_sum = idesc_h16_f32(128, S::kWideIn ? CO : 16, 1, 1, g.f16);
            const uint32_t w_lo = smem_desc_lo(smem_u32(wres), CO * 128);           // N blocks CO * 128 bytes apart
            const uint32_t ones_lo = smem_desc_lo(smem_u32(ones), 0), ones_hi = smem_desc_hi_sw128(0);
            uint32_t i = 0;
            bool ok = true;
            for (int t = tile_lo; t < tile_hi; ++t, ++i) {
                const uint32_t s = i & 1u, ph = (i >> 1) & 1u;
                const uint32_t buf = S::kDxBufs == 2 ? s : 0u, use = S::kDxBufs == 2 ? (i >> 1) : i;
                ok = mbar_wait_bounded(&ctl->dz_full[s], ph, abort_flag) &&
                     mbar_wait_bounded(&ctl->dx_empty[buf], (use & 1u) ^ 1u, abort_flag);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t dz_at = smem_u32(dz_tiles + (size_t)s * S::kDzBoxes * kPbBox);
                const uint32_t x_at = smem_u32(x_tiles + (size_t)s * S::kXBoxes * kPbBox);
                const uint32_t dz_k = smem_desc_lo(dz_at, 16), dz_mn = smem_desc_lo(dz_at, kPbBox), x_mn = smem_desc_lo(x_at, kPbBox);
                // dX tile = dZ tile x omega': K = C_out in steps of 16
                const uint32_t d_dx = tmem_base + buf * (uint32_t)CI;
#pragma unroll
                for (int kk = 0; kk < CO / 16; ++kk) {
                    const uint32_t a_lo = dz_k + (uint32_t)(kk >> 2) * kBox16 + (uint32_t)(kk & 3) * 2u, b_lo = w_lo + (uint32_t)kk * 128u;
                    if (kk == 0) umma_bf16_ss_halves<false>(d_dx, a_lo, hi, b_lo, hi, idesc_dx);
                    else umma_bf16_ss_halves<true>(d_dx, a_lo, hi, b_lo, hi, idesc_dx);
                }
                umma_commit(&ctl->dx_full[buf]);
                // domega' and sum dZ: K = the tile's 128 pixels in steps of 16 (two groups of 8 rows, 2048 bytes)
                const bool fresh = H ? i % kPbSegment == 0 : i == 0;
                ok = mbar_wait_bounded(&ctl->x_full[s], ph, abort_flag) &&
                     (!fresh || i == 0 || mbar_wait_bounded(&ctl->seg_empty, (i / kPbSegment - 1) & 1u, abort_flag));
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll 1
                for (int kt = 0; kt < 8; ++kt) {
                    const uint32_t koff = (uint32_t)kt * 128u;
                    const bool first = fresh && kt == 0;
#pragma unroll
                    for (int mb = 0; mb < S::kMBlocks; ++mb) {
                        const uint32_t d = tmem_base + (uint32_t)(S::kDwCol0 + mb * S::kNarrow);
                        const uint32_t a_lo = (S::kWideIn ? x_mn : dz_mn) + (uint32_t)(2 * mb) * kBox16 + koff;
                        const uint32_t b_lo = (S::kWideIn ? dz_mn : x_mn) + koff;
                        umma_bf16_ss_sel(d, a_lo, hi, b_lo, hi, idesc_dw, !first);
                        if (!S::kWideIn)
                            umma_bf16_ss_sel(tmem_base + (uint32_t)(S::kSumCol0 + mb * 16), a_lo, hi, ones_lo, ones_hi, idesc_sum, !first);
                    }
                    if (S::kWideIn)
                        umma_bf16_ss_sel(tmem_base + (uint32_t)S::kSumCol0, ones_lo, ones_hi, dz_mn + koff, hi, idesc_sum, !first);
                }
                umma_commit(&ctl->dz_empty[s]);
                umma_commit(&ctl->x_empty[s]);
                if (H && (i + 1) % kPbSegment == 0 && t + 1 < tile_hi) umma_commit(&ctl->seg_full);
            }
            if (ok) umma_commit(&ctl->acc_done);
            else give_up();
        }
    } else if (warp >= 10) {
        // ---- codes to X: this warp's 16 pixels of a tile, 16 codes a lane and turn ----
        constexpr int CHUNKS = CI / 16, TURNS = 16 * CHUNKS / 32;        // of 16 codes: a pixel's, a warp's per lane
        constexpr int AHEAD = TURNS < 8 ? TURNS : 8;                     // (8 at most: 256 channels)
        const int qw = warp - 10;
        uint4 next[AHEAD];
        uint32_t next_step[AHEAD];
        auto fetch = [&](int t) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int idx = a * 32 + lane, r = idx / CHUNKS, c = idx % CHUNKS;
                const long long pix = (long long)t * 128 + qw * 16 + r;
                next[a] = make_uint4(0u, 0u, 0u, 0u);                    // (past the last pixel: zeros, as dZ is)
                next_step[a] = 127u;
                if (pix < g.p) {
                    next[a] = __ldg((const uint4 *)(g.codes + (size_t)pix * CI + c * 16));
                    next_step[a] = __ldg(g.steps + (((size_t)pix * CI + c * 16) >> 5));
                }
            }
        };
        uint32_t i = 0;
        bool ok = true;
        if (tile_lo < tile_hi) fetch(tile_lo);
        for (int t = tile_lo; t < tile_hi; ++t, ++i) {
            const uint32_t s = i & 1u;
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->x_empty[s], ((i >> 1) & 1u) ^ 1u, abort_flag));
            if (!ok) break;
            uint8_t *tile = x_tiles + (size_t)s * S::kXBoxes * kPbBox;
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int idx = a * 32 + lane, r = qw * 16 + idx / CHUNKS, c = idx % CHUNKS;
                const float step = pack_step(next_step[a]);
                const f32x2 by = pair(step, step);
                const uint32_t word[4] = {next[a].x, next[a].y, next[a].z, next[a].w};
                uint32_t o[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    f32x2 f[2];
                    restore4(word[k], by, f);
                    o[2 * k] = narrow_t<H>(f[0]);
                    o[2 * k + 1] = narrow_t<H>(f[1]);
                }
                uint8_t *row = tile + (size_t)(c >> 2) * kPbBox + r * 128;
                const int c16 = (c & 3) * 2;
                *(uint4 *)(row + (((c16 ^ r) & 7) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                *(uint4 *)(row + ((((c16 + 1) ^ r) & 7) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
            }
            if (t + 1 < tile_hi) fetch(t + 1);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl->x_full[s]);
        }
        if (!ok && lane == 0) give_up();
    } else {
        // omega' = s omega (Sec. 3.3), one rounding, laid out as the MN-major B operand of the data-gradient GEMM: K = co rows of 128
        // bytes (64 ci), 128-byte swizzle, one block per 64 input channels
        for (int i = (int)threadIdx.x - 64; i < CO * (CI / 8); i += 256) {
            const int co = i / (CI / 8), c8 = i - co * (CI / 8), ci = c8 * 8;
            const float sc = g.vec3[co];
            const uint4 raw = __ldg((const uint4 *)(w + (size_t)co * CI + ci));
            const uint32_t in[4] = {raw.x, raw.y, raw.z, raw.w};
            uint32_t out[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                float lo, hi;
                unpack2_t<H>(in[h], lo, hi);
                out[h] = pack2_t<H>(lo * sc, hi * sc);
            }
            *(uint4 *)(wres + (size_t)(ci >> 6) * (CO * 128) + co * 128 + (((((ci & 63) >> 3) ^ (co & 7)) & 7) << 4)) =
                make_uint4(out[0], out[1], out[2], out[3]);
        }
        fence_proxy_async_smem();
        named_bar_sync(1, 288);
        // ---------------- epilogue ----------------
        const int quarter = warp & 3, ew = warp - 2, egroup = ew >> 2;
        uint8_t *boxes = staging + (size_t)ew * S::kOutBufs * kPbOut;
        uint64_t *add_bar = &ctl->add_full[ew];
        const uint32_t lane_sel = (uint32_t)(quarter * 32) << 16;
        const uint32_t frag_row = (uint32_t)((lane & 7) + (lane & 8)) * 128u, frag_chunk = (uint32_t)(((lane >> 4) ^ (lane & 7)) << 4);
        bool ok = true;
        uint32_t i = 0, turn = 0, add_ph = 0;
        for (int t = tile_lo; t <= tile_hi && ok; ++t, ++i) {
            const uint32_t s = i & 1u, buf = S::kDxBufs == 2 ? s : 0u, use = S::kDxBufs == 2 ? (i >> 1) : i;
            const bool last = t == tile_hi;
            if (last || (H && i && i % kPbSegment == 0)) {
                // ---- the CTA's partial of domega' as part[cta][co][ci] and its row of sums of dZ: 128 contiguous bytes per store, of later
                // segments added to what is there.  Both groups, before either waits for this tile: the issuer goes on when all eight
                // warps are through ----
                const bool more = H && i > kPbSegment;
                ok = __all_sync(0xffffffffu, last ? mbar_wait_bounded(&ctl->acc_done, 0, abort_flag)
                                                  : mbar_wait_bounded(&ctl->seg_full, (i / kPbSegment - 1) & 1u, abort_flag));
                if (last) pdl_launch_dependents();                     // (see umma_wgrad.cu)
                if (!ok) break;
                if (lane == 0) tma_store_wait_read<0>();               // (the boxes are free)
                __syncwarp();
                tc_fence_after_sync();
                float *part = partials + (size_t)blockIdx.x * CI * CO;
                // (added in L2, without a reading: each number has one thread, so the order is that of the segments)
                auto put = [&](float *at, uint32_t bits) {
                    if (more) atomicAdd(at, __uint_as_float(bits));
                    else *at = __uint_as_float(bits);
                };
                if (S::kWideIn) {
                    // accumulator row = ci (M block mb, lane), columns = co
                    for (int mb = egroup; mb < S::kMBlocks; mb += 2) {
                        float *ocol = part + mb * 128 + quarter * 32 + lane;
#pragma unroll 1
                        for (int c0 = 0; c0 < CO; c0 += 32) {
                            uint32_t v[32];
                            tmem_ld_32x32(tmem_base + (uint32_t)(S::kDwCol0 + mb * CO + c0) + lane_sel, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 32; ++j) put(ocol + (size_t)(c0 + j) * CI, v[j]);
                        }
                    }
                    if (warp == 2) {                               // every row of the sums tile is sum dZ: take this warp's first
                        float *brow = bsum + (size_t)blockIdx.x * CO;
#pragma unroll 1
                        for (int c0 = 0; c0 < CO; c0 += 32) {
                            uint32_t v[32];
                            tmem_ld_32x32(tmem_base + (uint32_t)(S::kSumCol0 + c0) + lane_sel, v);
                            tmem_ld_wait();
                            if (lane == 0) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) put(brow + c0 + j, v[j]);
                            }
                        }
                    }
                } else {
                    // accumulator row = co, columns = ci (64): 32 x 32 blocks are transposed in the warp's box (word (row, column) at row
                    // 32 + (column ^ row): no bank conflicts either way), then lane = ci
                    uint32_t *tr = (uint32_t *)boxes;
                    for (int mb = egroup; mb < S::kMBlocks; mb += 2) {
                        const int co0 = mb * 128 + quarter * 32;
#pragma unroll 1
                        for (int c0 = 0; c0 < CI; c0 += 32) {
                            uint32_t v[32];
                            int here = lane;
                            asm volatile("" : "+r"(here));    // (64 addresses that else are kept through all tiles)
                            tmem_ld_32x32(tmem_base + (uint32_t)(S::kDwCol0 + mb * CI + c0) + lane_sel, v);
                            tmem_ld_wait();
                            __syncwarp();
#pragma unroll
                            for (int j = 0; j < 32; ++j) tr[here * 32 + (j ^ here)] = v[j];
                            __syncwarp();
#pragma unroll 8
                            for (int r = 0; r < 32; ++r) put(part + (size_t)(co0 + r) * CI + c0 + lane, tr[r * 32 + (here ^ r)]);
                        }
                        uint32_t sv[16];
                        tmem_ld_32x16(tmem_base + (uint32_t)(S::kSumCol0 + mb * 16) + lane_sel, sv);
                        tmem_ld_wait();
                        put(bsum + (size_t)blockIdx.x * CO + co0 + lane, sv[0]);
                    }
                }
                if (last) break;
                tc_fence_before_sync();
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->seg_empty);
            }
            if (S::kDxBufs == 2 && (int)buf != egroup) continue;        // the two groups take alternate tiles ...
            // ... or halve the columns of the one accumulator
            const int c_lo = S::kDxBufs == 2 ? 0 : egroup * (CI / 2), c_hi = S::kDxBufs == 2 ? CI : c_lo + CI / 2;
            const int row0 = t * 128 + quarter * 32;
            auto box = [&]() { return boxes + (S::kOutBufs == 2 ? turn * kPbOut : 0u); };
            auto fetch_add = [&](int c0) {              // into the box whose last store has been read
                if (lane == 0) {
                    tma_store_wait_read<S::kOutBufs - 1>();
                    if (g.add) {
                        mbar_arrive_expect_tx(add_bar, kPbOut);
                        tma_load_2d(box(), &tm_add, add_bar, c0, row0);
                    }
                }
                __syncwarp();
            };
            fetch_add(c_lo);
            if (g.mask) ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->x_full[s], (i >> 1) & 1u, abort_flag));
            ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->dx_full[buf], use & 1u, abort_flag));
            if (!ok) {
                if (g.add) { if (lane == 0) mbar_wait_bounded(add_bar, add_ph, nullptr, 200000000ull); __syncwarp(); }
                break;
            }
            tc_fence_after_sync();
#pragma unroll 1
            for (int c0 = c_lo; c0 < c_hi; c0 += 64) {
                const uint32_t out = smem_u32(box()) + frag_row;
                const uint32_t xbox = smem_u32(x_tiles + ((size_t)s * S::kXBoxes + (c0 >> 6)) * kPbBox) + (uint32_t)quarter * kPbOut + frag_row;
                const uint32_t taddr = tmem_base + buf * (uint32_t)CI + (uint32_t)c0 + lane_sel;
                if (g.add) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(add_bar, add_ph, abort_flag));
                    if (!ok) {                          // (the copy in flight lands before the block ends)
                        if (lane == 0) mbar_wait_bounded(add_bar, add_ph, nullptr, 200000000ull);
                        __syncwarp();
                        break;
                    }
                    add_ph ^= 1u;
                }
                auto rows = [&](auto add_tag, auto mask_tag) {
                    constexpr bool ADD = decltype(add_tag)::value, MASK = decltype(mask_tag)::value;
#pragma unroll
                    for (int c = 0; c < 64; c += 32) {
                        uint32_t v[2][16];
                        tmem_ld_16x32(taddr + (uint32_t)c, v[0]);
                        tmem_ld_16x32(taddr + (16u << 16) + (uint32_t)c, v[1]);
                        tmem_ld_wait();
#pragma unroll
                        for (int q = 0; q < 4; q += 2)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                uint32_t r[4], a[4] = {0u, 0u, 0u, 0u}, m[4] = {0u, 0u, 0u, 0u};
                                const uint32_t at16 = (uint32_t)h * 2048u + (((uint32_t)(c / 8 + q) << 4) ^ frag_chunk);
                                if constexpr (ADD) ldmatrix_x4(a[0], a[1], a[2], a[3], out + at16);
                                if constexpr (MASK) ldmatrix_x4(m[0], m[1], m[2], m[3], xbox + at16);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const uint32_t *p2 = &v[h][(q + (e >> 1)) * 4 + (e & 1) * 2];
                                    f32x2 f = pair(__uint_as_float(p2[0]), __uint_as_float(p2[1]));
                                    if constexpr (ADD) f = fma2(f, pair(1.f, 1.f), widen_t<H>(a[e]));
                                    r[e] = post_pair<H>(narrow_t<H>(f), false, 0u, false, MASK, m[e]);
                                }
                                stmatrix_x4(out + at16, r[0], r[1], r[2], r[3]);
                            }
                    }
                };
                constexpr std::true_type yes{};
                constexpr std::false_type no{};
                if (g.add) { if (g.mask) rows(yes, yes); else rows(yes, no); }
                else { if (g.mask) rows(no, yes); else rows(no, no); }
                if (c0 + 64 >= c_hi) {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(&ctl->dx_empty[buf]); mbar_arrive(&ctl->x_empty[s]); }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    tma_store_2d(&tm_dx, box(), c0, row0);
                    tma_store_commit();
                }
                turn ^= 1u;
                if (c0 + 64 < c_hi) fetch_add(c0 + 64);
            }
        }
        if (lane == 0) tma_store_wait_all<0>();
        if (!ok && lane == 0) give_up();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, 512);
}

}  // namespace

// One CTA per SM, or, where accumulators are not emptied on the way, as many rounds of them as keep their sums short (1.56 M pixels
// 64 -> 128: two).
int packed_bwd1x1_ctas(const Problem &pb) {
    const long long tiles = (pb.p + 127) / 128, sms = device_sm_count(), most = sms * (kExactPixels / 128);
    const long long ctas = call_f16() ? sms : (tiles + most - 1) / most * sms;
    return (int)(tiles < ctas ? tiles : ctas);
}

cudaError_t launch_packed_bwd1x1(const Problem &pb, const void *dz, const void *codes, const void *steps, const void *w, const float *vec3,
                                 void *dx, float *partials, float *bsum, const void *add, bool mask, cudaStream_t st) {
    if (!fused_bwd1x1_eligible(pb)) return cudaErrorInvalidValue;
    PackedBwd g;
    g.p = pb.p; g.m_tiles = (int)((pb.p + 127) / 128); g.vec3 = vec3; g.f16 = call_f16();
    g.codes = (const uint8_t *)codes; g.steps = (const uint8_t *)steps;
    g.add = add != nullptr; g.mask = mask;
    CUtensorMap tdz, tdx, tadd;
    {   // a tile's [128 pixels][64 channels] blocks, side by side in shared memory, are one box
        const unsigned long long dims[3] = {64, (unsigned long long)pb.p, (unsigned long long)pb.c_out / 64};
        const unsigned long long str[3] = {0, (unsigned long long)pb.c_out * 2, 128};
        const unsigned int box[3] = {64, 128, (unsigned int)pb.c_out / 64};
        if (!make_tmap_tiled_bf16(&tdz, dz, 3, dims, str, box)) return cudaErrorInvalidValue;
    }
    if (!make_tmap_matrix_bf16(&tdx, dx, pb.p, pb.c_in, 32, 64)) return cudaErrorInvalidValue;
    tadd = tdx;
    if (add && !make_tmap_matrix_bf16(&tadd, add, pb.p, pb.c_in, 32, 64)) return cudaErrorInvalidValue;
    int *err = nullptr;
    if (cudaError_t e = error_word_address(&err); e != cudaSuccess) return e;
    auto go = [&](auto ci, auto co, auto half) {
        constexpr int CI = decltype(ci)::value, CO = decltype(co)::value;
        constexpr size_t smem = PbShape<CI, CO>::kSmem;
        auto kernel = packed_bwd1x1_kernel<CI, CO, decltype(half)::value>;
        static PerDevice attr, carve;
        if (cudaError_t e = max_dynamic_smem_once(kernel, 227 * 1024, &attr); e != cudaSuccess) return e;
        prefer_max_shared_once(kernel, &carve);
        return launch_pdl(kernel, dim3((unsigned)packed_bwd1x1_ctas(pb)), dim3(kPbThreads), smem, st, tdz, tdx, tadd, g,
                          (const __nv_bfloat16 *)w, partials, bsum, err);
    };
    auto typed = [&](auto ci, auto co) { return g.f16 ? go(ci, co, std::true_type()) : go(ci, co, std::false_type()); };
    using std::integral_constant;
    if (pb.c_in == 256) return typed(integral_constant<int, 256>(), integral_constant<int, 64>());
    if (pb.c_in == 128) return typed(integral_constant<int, 128>(), integral_constant<int, 64>());
    if (pb.c_out == 256) return typed(integral_constant<int, 64>(), integral_constant<int, 256>());
    return typed(integral_constant<int, 64>(), integral_constant<int, 128>());
}

}  // namespace convbn
