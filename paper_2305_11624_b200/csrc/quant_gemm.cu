// The deployed 8-bit product of rows that the kernel of quant_fused.cu does not take (more than 256 channels, ragged ones, wide results)
// and that are too many for quant_small.cu, as two kernels: rows to codes in the workspace, then a tensor-core GEMM of codes, both
// operands by TMA, 32-bit integer sums in tensor memory (kind::i8), the epilogue of quant8.cuh.
//
// GEMM: CTA = 10 warps: 0 loads, 1 MMA issuer and owner of tensor memory, 2-9 epilogue (two groups of four, an accumulator each).
// Persistent, tiles of 128 rows x BN channels dealt round-robin, the channel tiles of a row on neighbouring CTAs, so that codes
// come from L2 after their first reading.  PAIR: two CTAs share a 256 x BN product (cta_group::2), each brings its 128 rows and half of
// the channels: half the weight bytes into every SM.
// Bound by the MMAs (kind::i8 runs at twice the 16-bit rate), and in long runs by the power cap: 65536 rows 2048 -> 2048 166 us with the clock
// up, 3.3 POP/s, twice the measured 16-bit rate; 199 us at the 1.3 GHz of the cap.  The rows' pass in front of it, in which no MMA runs, takes
// 52 us: 230 us a call, 268 under the cap.
#include "kernels.h"
#include "quant8.cuh"

namespace convbn {

using namespace ptx;

namespace {

constexpr int kGThreads = 320;
constexpr int kGMaxStages = 8;
constexpr uint32_t kGABytes = 128 * 128;
constexpr uint32_t kGBox = 32 * 128;

struct QuantGemm {
    uint32_t p, tiles;             // rows; tiles (of a pair)
    int n, kb, tail, stages, dense, relu;      // tail: steps of 32 codes of the last block of 128
    FastDiv by_n;                  // channel tiles
};

struct GemmCtl {
    uint64_t full[kGMaxStages], empty[kGMaxStages], acc_full[2], acc_empty[2], add_full[8];
    uint32_t tmem_base;
    int abort_flag;
};

template <class T, int BN, bool PAIR>
__global__ void __launch_bounds__(kGThreads) quant_gemm_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w,
                                                               const __grid_constant__ CUtensorMap tm_z, const __grid_constant__ CUtensorMap tm_add,
                                                               const QuantGemm g, const float *__restrict__ xs, const float *__restrict__ ws,
                                                               const float *__restrict__ shift, const T *__restrict__ add,
                                                               T *__restrict__ z, int *err) {
    extern __shared__ uint8_t smem_raw[];
    constexpr int CTAS = PAIR ? 2 : 1;
    constexpr uint32_t kWBytes = BN / CTAS * 128, kStage = kGABytes + kWBytes;
    uint8_t *tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *staging = tiles + (size_t)g.stages * kStage;                    // 8 warps x [32 rows][128 bytes]
    float *params = (float *)(staging + 8 * kGBox);                          // 2 groups x [scale BN | shift BN]
    GemmCtl *ctl = (GemmCtl *)(params + 4 * BN);
    const uint32_t rank = PAIR ? cluster_rank() : 0u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &ctl->abort_flag;
    // tile t: its first row and channel (of an odd number of row tiles the last has no partner: all rows out of range)
    auto tile_of = [&](uint32_t i, uint32_t &row0, int &n0) -> bool {
        const uint32_t t = blockIdx.x / CTAS + i * (gridDim.x / CTAS);
        if (t >= g.tiles) return false;
        const uint32_t mt = g.by_n.div(t);
        n0 = (int)(t - mt * g.by_n.d) * BN;
        row0 = (mt * CTAS + rank) * 128u;
        return true;
    };
    auto give_up = [&]() { atomicOr(err, ERRW_TIMEOUT); ctl->abort_flag = 1; };

    if (threadIdx.x == 64) { prefetch_tensormap(&tm_x); prefetch_tensormap(&tm_w); }
    if (threadIdx.x == 96) {
        for (int s = 0; s < kGMaxStages; ++s) { mbar_init(&ctl->full[s], 1); mbar_init(&ctl->empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&ctl->acc_full[a], 1); mbar_init(&ctl->acc_empty[a], 4 * CTAS); }
        for (int a = 0; a < 8; ++a) mbar_init(&ctl->add_full[a], 1);
        ctl->abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc<CTAS>(&ctl->tmem_base, 2 * BN);
        tmem_relinquish<CTAS>();
    }
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();
    tc_fence_after_sync();
    pdl_wait();
    pdl_launch_dependents();
    const uint32_t tmem_base = ctl->tmem_base;
    const uint32_t sb_end = 8u * (uint32_t)g.stages;

    if (warp == 0) {
        if (elect_one()) {
            // a pair's boxes all count on its first CTA's barriers
            const uint32_t full0 = PAIR ? cluster_addr(&ctl->full[0], 0) : smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);
            const uint32_t tiles0 = smem_u32(tiles);
            uint32_t it = 0, sb = 0, slot = tiles0, ph = 1, row0;
            int n0;
            bool ok = true, free = false;
            for (uint32_t i = 0; ok && tile_of(i, row0, n0); ++i) {
#pragma unroll 2
                for (int kb = 0; kb < g.kb; ++kb) {
                    if (!free) ok = mbar_wait_bounded(empty0 + sb, ph, abort_flag);
                    if (!ok) break;
                    const uint32_t bar = full0 + sb, dst = slot;
                    ++it; sb += 8; slot += kStage;
                    if (sb == sb_end) { sb = 0; slot = tiles0; ph ^= 1u; }
                    free = mbar_test_wait(empty0 + sb, ph);
                    if (rank == 0) mbar_arrive_expect_tx(bar, CTAS * kStage);
                    if constexpr (PAIR) {
                        tma_load_2d_pair(dst, &tm_x, bar, kb * 128, (int)row0);
                        tma_load_2d_pair(dst + kGABytes, &tm_w, bar, kb * 128, n0 + (int)rank * (BN / 2));
                    } else {
                        tma_load_2d(dst, &tm_x, bar, kb * 128, (int)row0);
                        tma_load_2d(dst + kGABytes, &tm_w, bar, kb * 128, n0);
                    }
                }
            }
            // the first CTA's commits arrive in the second too: seen here before its CTA may exit
            if constexpr (PAIR)
                for (uint32_t j = it > (uint32_t)g.stages ? it - g.stages : 0; ok && j < it; ++j)
                    ok = mbar_wait_bounded(&ctl->empty[j % g.stages], (j / g.stages) & 1u, abort_flag);
            if (!ok) {
                give_up();
                if constexpr (PAIR) {     // counted in the first CTA as far as that has got: a millisecond is ample for any of them
                    for (const uint64_t t0 = globaltimer_ns(); globaltimer_ns() - t0 < 1000000ull;) {}
                } else {
                    for (uint32_t j = it > (uint32_t)g.stages ? it - g.stages : 0; j < it; ++j)      // let the copies in flight land
                        mbar_wait_bounded(&ctl->full[j % g.stages], (j / g.stages) & 1u, nullptr, 200000000ull);
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = idesc_s8(128 * CTAS, BN), hi = smem_desc_hi_sw128(1024);
            const uint32_t tiles_lo = smem_desc_lo(smem_u32(tiles), 16), full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);
            auto commit = [](auto bar) {
                if constexpr (PAIR) umma_commit_pair(bar); else umma_commit(bar);
            };
            uint32_t sb = 0, ph = 0, a_lo = tiles_lo, row0;
            int n0;
            bool ok = true, ready = false;
            for (uint32_t i = 0; ok && tile_of(i, row0, n0); ++i) {
                const uint32_t acc = i & 1u, d = tmem_base + acc * BN;
                ok = mbar_wait_bounded(&ctl->acc_empty[acc], ((i >> 1) & 1u) ^ 1u, abort_flag);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll 2
                for (int kb = 0; kb < g.kb; ++kb) {
                    if (!ready && !mbar_wait_bounded(full0 + sb, ph, abort_flag)) { ok = false; break; }
                    const uint32_t a0 = a_lo, w0 = a_lo + (kGABytes >> 4), done = empty0 + sb;
                    sb += 8; a_lo += kStage >> 4;
                    if (sb == sb_end) { sb = 0; a_lo = tiles_lo; ph ^= 1u; }
                    ready = mbar_test_wait(full0 + sb, ph);
                    const int steps = kb + 1 == g.kb ? g.tail : 4;
                    umma_s8<CTAS>(d, a0, hi, w0, hi, idesc, (uint32_t)kb);
                    for (int q = 1; q < steps; ++q) umma_s8<CTAS>(d, a0 + 2u * q, hi, w0 + 2u * q, hi, idesc, 1u);
                    commit(done);
                }
                if (ok) commit(&ctl->acc_full[acc]);
            }
            if (!ok) give_up();
        }
    } else {
        constexpr int CH = 128 / sizeof(T);
        const int quarter = warp & 3, ew = warp - 2;
        const uint32_t egroup = (uint32_t)ew >> 2;
        uint8_t *buf = staging + (size_t)ew * kGBox;
        float *scale_s = params + egroup * 2 * BN, *shift_s = scale_s + BN;
        uint64_t *add_bar = &ctl->add_full[ew];
        const QuantOut<T> out{z, add, g.p, g.n, g.dense, g.relu};
        const bool boxed = g.dense && add;
        bool ok = true;
        uint32_t row0, add_ph = 0;
        int n0;
        for (uint32_t i = 0; ok && tile_of(i, row0, n0); ++i) {
            if ((i & 1u) != egroup) continue;
            row0 += quarter * 32;
            const int cols = min(BN, g.n - n0);
            auto fetch_add = [&](int c0) {              // into the box whose last store has been read
                if (lane == 0) {
                    tma_store_wait_read<0>();
                    if (boxed) {
                        mbar_arrive_expect_tx(add_bar, kGBox);
                        tma_load_2d(buf, &tm_add, add_bar, n0 + c0, (int)row0);
                    }
                }
                __syncwarp();
            };
            if (g.dense) fetch_add(0);
            // this group's channels (its last readers are past the barrier below, of the tile before)
            named_bar_sync(1 + egroup, 128);
            for (int c = (int)(threadIdx.x & 127u); c < BN; c += 128) {
                scale_s[c] = n0 + c < g.n ? __ldg(ws + n0 + c) : 0.f;
                shift_s[c] = n0 + c < g.n ? __ldg(shift + n0 + c) : 0.f;
            }
            f32x2 xs2[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t row = row0 + (g.dense && sizeof(T) == 2 ? lane / 4 + 8 * k : lane);
                const float v = row < g.p ? __ldg(xs + row) : 0.f;
                xs2[k] = pair(v, v);
            }
            named_bar_sync(1 + egroup, 128);
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->acc_full[i & 1u], (i >> 1) & 1u, abort_flag));
            if (!ok) {
                if (boxed) { if (lane == 0) mbar_wait_bounded(add_bar, add_ph, nullptr, 200000000ull); __syncwarp(); }
            }
            tc_fence_after_sync();
            const uint32_t t_row = tmem_base + (i & 1u) * BN + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
            for (int c0 = 0; ok && c0 < cols; c0 += CH) {
                if (boxed) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(add_bar, add_ph, abort_flag));
                    if (!ok) {                              // (the copy in flight lands before the block ends)
                        if (lane == 0) mbar_wait_bounded(add_bar, add_ph, nullptr, 200000000ull);
                        __syncwarp();
                        break;
                    }
                    add_ph ^= 1u;
                }
                quant_chunk<T, false>(out, buf, boxed, t_row + (uint32_t)c0, scale_s + c0, shift_s + c0, xs2, row0 + lane, n0 + c0, cols - c0, lane);
                if (c0 + CH >= cols) {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (PAIR) mbar_arrive_cluster(cluster_addr(&ctl->acc_empty[i & 1u], 0));
                        else mbar_arrive(&ctl->acc_empty[i & 1u]);
                    }
                }
                if (g.dense) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(&tm_z, buf, n0 + c0, (int)row0);
                        tma_store_commit();
                    }
                    if (c0 + CH < cols) fetch_add(c0 + CH);
                }
            }
            // (the warps of a group give up together: the barriers above are for all four)
            ok = named_bar_all(1 + egroup, 128, ok);
        }
        if (!ok && lane == 0) give_up();
        if (lane == 0) tma_store_wait_all<0>();
    }
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();
    if (warp == 1) tmem_dealloc<CTAS>(tmem_base, 2 * BN);
}

// Rows to codes.  LPR lanes a row, KEEP chunks of eight elements a lane kept from the search for the largest magnitude to the codes
// (what lies beyond is read again, from L1 or L2); short rows several to a lane, so that a warp has at least four requests out.
// (16384 rows of 2048 bf16 15.9 us: 67 MB read and 34 written at the memory's rate.)
template <class T, int LPR, int KEEP, bool VEC>
__global__ void __launch_bounds__(256) quant_rows_kernel(const RowMap rows, uint32_t p, int k, int pitch, const T *__restrict__ x,
                                                         uint8_t *__restrict__ codes, float *__restrict__ scale) {
    constexpr int RPI = 32 / LPR, SETS = KEEP < 4 ? 4 / KEEP : 1;
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, sub = lane & (LPR - 1);
    const uint32_t first = (blockIdx.x * 8 + (threadIdx.x >> 5)) * (RPI * SETS) + lane / LPR;
    auto read = [&](Eight<T> &v, const T *src, int at) {
        if (at >= k) v.zero();
        else if constexpr (VEC) v.load(src + at);
        else v.load_some(src + at, k - at);
    };
    Eight<T> kept[SETS][KEEP];
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        const T *src = x + rows.at(min(first + s * RPI, p - 1));
#pragma unroll
        for (int c = 0; c < KEEP; ++c) read(kept[s][c], src, (c * LPR + sub) * 8);
    }
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        const uint32_t row = first + s * RPI;
        const T *src = x + rows.at(min(row, p - 1));
        uint32_t top = kept[s][0].top();
#pragma unroll
        for (int c = 1; c < KEEP; ++c) top = max(top, kept[s][c].top());
        if constexpr (LPR == 32)
            for (int at = (KEEP * 32 + lane) * 8; at < k; at += 256) {
                Eight<T> v;
                read(v, src, at);
                top = max(top, v.top());
            }
        if constexpr (LPR == 32) top = __reduce_max_sync(0xffffffffu, top);
        else
#pragma unroll
            for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const RowScale rs = row_scale(Eight<T>::top_f32(top));
        if (row >= p) continue;
        uint8_t *dst = codes + (size_t)row * pitch;
#pragma unroll
        for (int c = 0; c < KEEP; ++c)
            if ((c * LPR + sub) * 8 < pitch) *(uint2 *)(dst + (c * LPR + sub) * 8) = kept[s][c].codes(rs.inv);
        if constexpr (LPR == 32)
            for (int at = (KEEP * 32 + lane) * 8; at < pitch; at += 256) {
                Eight<T> v;
                read(v, src, at);
                *(uint2 *)(dst + at) = v.codes(rs.inv);
            }
        if (sub == 0) scale[row] = rs.scale;
    }
}

template <class T, int BN, bool PAIR>
cudaError_t launch_gemm(const Problem &pb, const void *xq, const float *xs, const void *wq, const float *ws, const float *shift,
                        const void *add, int relu, void *z, int *err, cudaStream_t st) {
    constexpr int CTAS = PAIR ? 2 : 1;
    const int sms = device_sm_count(), es = (int)sizeof(T);
    QuantGemm g;
    g.p = (uint32_t)pb.p; g.n = pb.c_out; g.relu = relu;
    g.kb = (pb.c_in + 127) / 128; g.tail = (pb.c_in - (g.kb - 1) * 128 + 31) / 32;
    g.dense = (size_t)pb.c_out * es % 16 == 0;
    const long long n_tiles = (pb.c_out + BN - 1) / BN, m_tiles = (pb.p + 128 * CTAS - 1) / (128 * CTAS);
    if (n_tiles * m_tiles >= (1LL << 31)) return cudaErrorInvalidValue;
    g.tiles = (uint32_t)(n_tiles * m_tiles);
    g.by_n = FastDiv((uint32_t)n_tiles);
    const size_t stage = kGABytes + BN / CTAS * 128, fixed = 1024 + 8 * kGBox + 16 * BN + sizeof(GemmCtl) + 16;
    int stages = (int)((226 * 1024 - fixed) / stage);
    g.stages = stages > kGMaxStages ? kGMaxStages : stages;
    CUtensorMap tx, tw, tz, ta;
    if (!make_tmap_matrix_bytes(&tx, xq, pb.p, quant_pitch(pb), 1, 128) ||
        !make_tmap_matrix_bytes(&tw, wq, pb.c_out, quant_pitch(pb), 1, BN / CTAS))
        return cudaErrorInvalidValue;
    tz = ta = tw;
    if (g.dense) {
        if (!make_tmap_matrix_bytes(&tz, z, pb.p, pb.c_out, es, 32)) return cudaErrorInvalidValue;
        if (add && !make_tmap_matrix_bytes(&ta, add, pb.p, pb.c_out, es, 32)) return cudaErrorInvalidValue;
    }
    const uint32_t slots = (uint32_t)(sms / CTAS), grid = (g.tiles < slots ? g.tiles : slots) * CTAS;
    static PerDevice attr, carve;
    auto kernel = quant_gemm_kernel<T, BN, PAIR>;
    if (cudaError_t e = max_dynamic_smem_once(kernel, 227 * 1024, &attr); e != cudaSuccess) return e;
    prefer_max_shared_once(kernel, &carve);
    return launch_pdl<CTAS>(kernel, dim3(grid), dim3(kGThreads), g.stages * stage + fixed, st, tx, tw, tz, ta, g, xs, ws, shift, (const T *)add,
                            (T *)z, err);
}

}  // namespace

cudaError_t launch_quant_rows(const Problem &pb, int dtype, const void *x, void *codes, float *scale, cudaStream_t st) {
    const RowMap rows = quant_row_map(pb);
    auto sized = [&](auto tag, auto lpr, auto keep) {
        using T = decltype(tag);
        constexpr int LPR = decltype(lpr)::value, KEEP = decltype(keep)::value, PER = 8 * (32 / LPR) * (KEEP < 4 ? 4 / KEEP : 1);
        auto kernel = pb.c_in % 8 == 0 ? quant_rows_kernel<T, LPR, KEEP, true> : quant_rows_kernel<T, LPR, KEEP, false>;
        return launch_pdl(kernel, dim3((unsigned)((pb.p + PER - 1) / PER)), dim3(256), 0, st, rows, (uint32_t)pb.p, pb.c_in, quant_pitch(pb),
                          (const T *)x, (uint8_t *)codes, scale);
    };
    auto go = [&](auto tag) {
        using std::integral_constant;
        if (pb.c_in <= 64) return sized(tag, integral_constant<int, 8>(), integral_constant<int, 1>());
        if (pb.c_in <= 128) return sized(tag, integral_constant<int, 16>(), integral_constant<int, 1>());
        if (pb.c_in <= 256) return sized(tag, integral_constant<int, 32>(), integral_constant<int, 1>());
        if (pb.c_in <= 512) return sized(tag, integral_constant<int, 32>(), integral_constant<int, 2>());
        if (pb.c_in <= 1024) return sized(tag, integral_constant<int, 32>(), integral_constant<int, 4>());
        return sized(tag, integral_constant<int, 32>(), integral_constant<int, 8>());
    };
    return dtype == CONVBN_F32 ? go(float()) : (dtype == CONVBN_F16 ? go(__half()) : go(__nv_bfloat16()));
}

cudaError_t launch_quant_gemm(const Problem &pb, int dtype, const void *xq, const float *xs, const void *wq, const float *ws,
                              const float *shift, const void *add, int relu, void *z, cudaStream_t st) {
    int *err = nullptr;
    if (cudaError_t e = error_word_address(&err); e != cudaSuccess) return e;
    // Wide tiles of pairs where they fill the SMs twice; otherwise the width that leaves the fewest SMs idle.
    const long long sms = device_sm_count(), m = (pb.p + 127) / 128;
    const long long pairs = (m + 1) / 2 * ((pb.c_out + 255) / 256);
    auto go = [&](auto tag) {
        using T = decltype(tag);
        if (pairs >= sms) return launch_gemm<T, 256, true>(pb, xq, xs, wq, ws, shift, add, relu, z, err, st);
        if (m * ((pb.c_out + 127) / 128) >= sms) return launch_gemm<T, 128, false>(pb, xq, xs, wq, ws, shift, add, relu, z, err, st);
        return launch_gemm<T, 64, false>(pb, xq, xs, wq, ws, shift, add, relu, z, err, st);
    };
    return dtype == CONVBN_F32 ? go(float()) : (dtype == CONVBN_F16 ? go(__half()) : go(__nv_bfloat16()));
}

}  // namespace convbn
