// The deployed 1x1 block in 8-bit integers as ONE kernel (convbn_deploy_fwd_quant): rows of X become codes on their way into shared
// memory, the product runs on the tensor cores (tcgen05, 8-bit operands, 32-bit integer sums in tensor memory), scales, shift,
// addend and ReLU are applied to the sums.  X is read once in its storage type, Z written once; codes exist on chip only.
//
// CTA = 19 warps: 0 weight tiles (TMA), 1 MMA issuer and owner of tensor memory, 2-9 epilogue (two groups of four, an accumulator
// each), 10-17 rows to codes, 18 brings the rows by TMA into a ring.  A unit of work is 128 rows: they are read whole, a row by 8, 16 or
// 32 lanes, for their largest magnitudes and again for the codes, which are written as the K-major A operand (128-byte swizzle).
// Bound by those two readings for long rows, by the epilogue for wide outputs: 256 -> 64 at 56 x 56, N = 256 109 us (78.5 at the
// measured copy bandwidth), 64 -> 256, N = 128 56.1 (39.3), 128 -> 128, N = 128 41.7 (31.4).
#include "kernels.h"
#include "quant8.cuh"

namespace convbn {

using namespace ptx;

namespace {

constexpr int kQRows = 128;                      // rows of a unit (UMMA M)
constexpr uint32_t kQBlock = kQRows * 128;       // [128 rows][128 codes] of the A operand
constexpr int kQThreads = 608;
constexpr int kQLoadWarp = 10;                   // first of the eight warps that make codes
constexpr int kQRowWarp = 18;                    // brings the rows
constexpr int kQMaxStages = 8;
constexpr uint32_t kQStage = 32 * 128;           // an epilogue warp's box: [32 rows][128 bytes]
constexpr int kQSlots = 4;                       // row scales of so many units
constexpr int kQMaxDepth = 8;                    // slots of a ring of rows

struct QuantFused {
    int strided, stride_h, stride_w;             // rows of X that are not side by side: im2col boxes
    FastDiv by_w, by_h;                          // output extent
    int boxes;                                   // of 128 bytes of a row of X
    uint32_t p;
    int k, kb, n, bn;                            // C_in, its blocks of 128, C_out, channels of a tile
    uint32_t units, n_tiles;
    int stages, nbuf, resident;                  // slots of streamed weights, boxes of an epilogue warp
    int rings, depth;                            // rings of rows (one per converting group), their slots
    int dense, relu;                             // rows of Z start on 16-byte boundaries
};

struct QuantCtl {
    uint64_t rows_full[2][kQMaxDepth], rows_empty[2][kQMaxDepth], full[kQMaxStages], empty[kQMaxStages], wfull, a_full[2], a_empty[2];
    uint64_t xs_full[kQSlots], acc_full[2], acc_empty[2], add_full[8];
    uint32_t tmem_base;
    int abort_flag;
};

// The eight converting warps work on a unit together, or, rows of up to 64 elements, in two groups that take the units in turn (GROUPS).
// A warp has ROWS of its group's units, RPI of them an instruction (a set), BATCH sets at a time, at most 4 KB.  Half a batch of a group's
// warps, side by side, is a slot of the group's ring.
template <class T, int LPR> struct RowSets {
    static constexpr int GROUPS = LPR == 8 ? 2 : 1, WARPS = 8 / GROUPS, ROWS = kQRows / WARPS;
    static constexpr int RPI = 32 / LPR, SETS = ROWS / RPI, SET_BYTES = 256 * (int)sizeof(T);
    static constexpr int BATCH = SETS * SET_BYTES <= 4096 ? SETS : 4096 / SET_BYTES, BATCHES = SETS / BATCH, HALF = BATCH / 2;
    static constexpr int SLOT_ROWS = WARPS * HALF * RPI;
    static constexpr uint32_t SLOT_BYTES = (uint32_t)(WARPS * HALF * SET_BYTES);
};

// LPR lanes read a row, eight elements each.
template <class T, int LPR>
__global__ void __launch_bounds__(kQThreads) quant_fused_kernel(const __grid_constant__ CUtensorMap tm_x,
                                                                const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_z,
                                                                const __grid_constant__ CUtensorMap tm_add, const QuantFused g,
                                                                const float *__restrict__ ws,
                                                                const float *__restrict__ shift, const T *__restrict__ add,
                                                                T *__restrict__ z, int *err) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *a_tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t a_bytes = (uint32_t)g.kb * kQBlock, w_bytes = (uint32_t)g.bn * 128;
    uint8_t *w_tiles = a_tiles + 2 * (size_t)a_bytes;
    uint8_t *staging = w_tiles + (size_t)(g.resident ? g.n_tiles * g.kb : g.stages) * w_bytes;
    uint8_t *ring = staging + (size_t)8 * g.nbuf * kQStage;
    float *scale_s = (float *)(ring + RowSets<T, LPR>::GROUPS * (size_t)g.depth * RowSets<T, LPR>::SLOT_BYTES), *shift_s = scale_s + g.n_tiles * g.bn;
    float *xs_s = shift_s + g.n_tiles * g.bn;                                   // [kQSlots][128]
    QuantCtl *ctl = (QuantCtl *)(xs_s + kQSlots * kQRows);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &ctl->abort_flag;

    if (threadIdx.x == 0) {
        prefetch_tensormap(&tm_x); prefetch_tensormap(&tm_w);
        for (int s = 0; s < kQMaxStages; ++s) { mbar_init(&ctl->full[s], 1); mbar_init(&ctl->empty[s], 1); }
        mbar_init(&ctl->wfull, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(&ctl->a_full[s], RowSets<T, LPR>::WARPS); mbar_init(&ctl->a_empty[s], 1);
            mbar_init(&ctl->acc_full[s], 1); mbar_init(&ctl->acc_empty[s], 4);
        }
        for (int s = 0; s < kQSlots; ++s) mbar_init(&ctl->xs_full[s], RowSets<T, LPR>::WARPS);
        for (int s = 0; s < 8; ++s) {
            mbar_init(&ctl->add_full[s], 1);
        }
        for (int s = 0; s < 2 * kQMaxDepth; ++s) {
            mbar_init(&ctl->rows_full[0][0] + s, 1);
            mbar_init(&ctl->rows_empty[0][0] + s, RowSets<T, LPR>::WARPS);
        }
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

    if (warp == 0) {
        if (elect_one()) {
            bool ok = true;
            uint32_t it = 0;
            if (g.resident) {
                mbar_arrive_expect_tx(&ctl->wfull, g.n_tiles * g.kb * w_bytes);
                for (uint32_t nt = 0; nt < g.n_tiles; ++nt)
                    for (int kb = 0; kb < g.kb; ++kb)
                        tma_load_2d(w_tiles + (size_t)(nt * g.kb + kb) * w_bytes, &tm_w, &ctl->wfull, kb * 128, (int)nt * g.bn);
            } else {
                for (uint32_t u = blockIdx.x; ok && u < g.units; u += gridDim.x)
                    for (uint32_t nt = 0; ok && nt < g.n_tiles; ++nt)
                        for (int kb = 0; kb < g.kb; ++kb, ++it) {
                            const uint32_t s = it % g.stages, ph = (it / g.stages) & 1u;
                            ok = mbar_wait_parked(&ctl->empty[s], ph ^ 1u, abort_flag);
                            if (!ok) break;
                            mbar_arrive_expect_tx(&ctl->full[s], w_bytes);
                            tma_load_2d(w_tiles + (size_t)s * w_bytes, &tm_w, &ctl->full[s], kb * 128, (int)nt * g.bn);
                        }
            }
            if (!ok) {
                give_up();
                for (uint32_t j = it > (uint32_t)g.stages ? it - g.stages : 0; j < it; ++j)      // let the copies in flight land
                    mbar_wait_parked(&ctl->full[j % g.stages], (j / g.stages) & 1u, nullptr, 200000000ull);
            } else if (g.resident) {
                mbar_wait_parked(&ctl->wfull, 0, nullptr, 200000000ull);
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t idesc = idesc_s8(kQRows, g.bn), hi = smem_desc_hi_sw128(1024);
            const uint32_t a0 = smem_desc_lo(smem_u32(a_tiles), 16), w0 = smem_desc_lo(smem_u32(w_tiles), 16);
            const int tail = (g.k - (g.kb - 1) * 128 + 31) / 32;              // steps of 32 codes of the last block
            bool ok = !g.resident || mbar_wait_parked(&ctl->wfull, 0, abort_flag);
            uint32_t i = 0, s = 0, it = 0;
            for (uint32_t u = blockIdx.x; ok && u < g.units; u += gridDim.x, ++i) {
                const uint32_t ab = i & 1u, use = i >> 1;
                ok = mbar_wait_parked(&ctl->a_full[ab], use & 1u, abort_flag);
                for (uint32_t nt = 0; ok && nt < g.n_tiles; ++nt, ++s) {
                    const uint32_t acc = s & 1u, d = tmem_base + acc * (uint32_t)g.bn;
                    ok = mbar_wait_parked(&ctl->acc_empty[acc], ((s >> 1) & 1u) ^ 1u, abort_flag);
                    if (!ok) break;
                    tc_fence_after_sync();
                    for (int kb = 0; kb < g.kb; ++kb) {
                        uint32_t slot = nt * g.kb + kb;
                        if (!g.resident) {
                            slot = it % g.stages;
                            ok = mbar_wait_parked(&ctl->full[slot], (it / g.stages) & 1u, abort_flag);
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
                if (ok && u + 2 * gridDim.x < g.units) umma_commit(&ctl->a_empty[ab]);
            }
            if (!ok) give_up();
        }
    } else if (warp == kQRowWarp) {
        // ---- rows of X, a slot at a time, into the ring of the group that converts the unit: boxes of [SLOT_ROWS][128 bytes] ----
        using R = RowSets<T, LPR>;
        constexpr int COLS = 128 / sizeof(T);                 // columns of a box
        uint32_t asked[2] = {0, 0}, i = 0;
        bool ok = true;
        if (elect_one()) {
            for (uint32_t u = blockIdx.x; ok && u < g.units; u += gridDim.x, ++i) {
                const uint32_t end = min((u + 1) * kQRows, g.p), qg = R::GROUPS == 2 ? i & 1u : 0u;
                for (uint32_t first = u * kQRows; first < end; first += R::SLOT_ROWS) {
                    const uint32_t n = qg ? asked[1] : asked[0], turn = n / (uint32_t)g.depth, slot = n - turn * (uint32_t)g.depth;
                    uint64_t *full = &ctl->rows_full[qg][slot];
                    ok = mbar_wait_parked(&ctl->rows_empty[qg][slot], (turn & 1u) ^ 1u, abort_flag);
                    if (!ok) break;
                    uint8_t *to = ring + ((size_t)qg * g.depth + slot) * R::SLOT_BYTES;
                    mbar_arrive_expect_tx(full, (uint32_t)g.boxes * (R::SLOT_ROWS * 128));
                    int img = 0, ho = 0, wo = 0;
                    if (g.strided) {
                        const uint32_t t = g.by_w.div(first);
                        img = (int)g.by_h.div(t);
                        ho = (int)(t - (uint32_t)img * g.by_h.d) * g.stride_h;
                        wo = (int)(first - t * g.by_w.d) * g.stride_w;
                    }
                    for (int c = 0; c < g.boxes; ++c, to += R::SLOT_ROWS * 128) {
                        if (g.strided) tma_load_im2col_4d(to, &tm_x, full, c * COLS, wo, ho, img, 0, 0);
                        else tma_load_2d(to, &tm_x, full, c * COLS, (int)first);
                    }
                    if (qg) ++asked[1]; else ++asked[0];
                }
            }
        }
        if (!ok) {                                            // (the thread that asked)
            give_up();
            for (int qg = 0; qg < 2; ++qg)
                for (uint32_t j = asked[qg] > (uint32_t)g.depth ? asked[qg] - g.depth : 0; j < asked[qg]; ++j)    // let the copies in flight land
                    mbar_wait_parked(&ctl->rows_full[qg][j % g.depth], (j / g.depth) & 1u, nullptr, 200000000ull);
        }
    } else if (warp >= kQLoadWarp) {
        // ---- rows to codes ----
        // What a unit costs beside its elements (waits, scales, the hand-over) is most of it where rows are short: two groups, each with an A
        // buffer of its own, halve that and run beside each other, 64 -> 64 at 56 x 56, N = 256 62 -> 51 us; longer rows want the ring in
        // one piece, 256 -> 64 132 us and 157 by groups (sixteen warps in two groups: 133 where eight in one took 118; all of these before
        // row addresses were formed once and waiting warps parked, which took 118 to 109).  A batch's rows are
        // read twice: for their largest magnitudes, and after these have become scales, which each lane works out for one row (a scale
        // per four rows, and the rows kept in registers between: 192 us).
        using R = RowSets<T, LPR>;
        constexpr int RPI = R::RPI, BATCH = R::BATCH, BATCHES = R::BATCHES, HALF = R::HALF, SLOT_ROWS = R::SLOT_ROWS;
        const int qg = R::GROUPS == 2 ? (warp - kQLoadWarp) >> 2 : 0, qw = (warp - kQLoadWarp) & (R::WARPS - 1);
        const int sub = lane & (LPR - 1), row_l = lane / LPR, own = qw * HALF * RPI + row_l;     // row in a slot
        const uint32_t ring0 = smem_u32(ring) + (uint32_t)(qg * g.depth) * RowSets<T, LPR>::SLOT_BYTES;
        uint32_t slot = 0, ph = 0;
        // Where set j of a half batch is for this lane, in its slot and in its unit's A operand (slots and their rows in the unit start on
        // multiples of eight rows).  Formed for every row anew, from pointers whose kind the compiler cannot see, these took as many
        // instructions as all else.
        uint32_t from[HALF], to[HALF];
#pragma unroll
        for (int j = 0; j < HALF; ++j) {
            const uint32_t r = (uint32_t)(own + j * RPI), chunk = (uint32_t)sub * (sizeof(T) / 2), at = (uint32_t)sub * 8u;
            from[j] = (chunk >> 3) * (SLOT_ROWS * 128) + r * 128u + (((chunk ^ r) & 7u) << 4);
            to[j] = (at >> 7) * kQBlock + r * 128u + ((((at >> 4) ^ r) & 7u) << 4) + (at & 8u);
        }
        const bool there_is = sub * 8 < g.boxes * (int)(128 / sizeof(T));                          // (a box with these elements)
        auto read = [&](Eight<T> &v, uint32_t at) { if (there_is) v.load_shared(at); else v.zero(); };
        // set j of a batch in its unit
        auto row_of = [&](int batch, int j) { return (2 * batch + j / HALF) * SLOT_ROWS + own + j % HALF * RPI; };
        bool ok = true;
        uint32_t i = 0;
        for (uint32_t u = blockIdx.x; ok && u < g.units; u += gridDim.x, ++i) {
            const uint32_t ab = i & 1u, use = i >> 1;
            if (R::GROUPS == 2 && (int)ab != qg) continue;    // (the other group's)
            const uint32_t tile = smem_u32(a_tiles) + ab * a_bytes, xs = smem_u32(xs_s) + (i % kQSlots) * (kQRows * 4u);
            const uint32_t first = u * kQRows;
#pragma unroll 1
            for (int batch = 0; batch < BATCHES; ++batch) {
                uint32_t t[BATCH], base[2], bar[2];
                bool there[2];
#pragma unroll
                for (int j = 0; j < BATCH; ++j) t[j] = 0u;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    there[h] = first + (uint32_t)((2 * batch + h) * SLOT_ROWS) < g.p;       // (a slot past the last row never comes)
                    base[h] = ring0 + slot * RowSets<T, LPR>::SLOT_BYTES;
                    bar[h] = slot;
                    if (!there[h]) continue;
                    ok = __all_sync(0xffffffffu, mbar_wait_parked(&ctl->rows_full[qg][slot], ph, abort_flag));
                    if (!ok) break;
                    if (++slot == (uint32_t)g.depth) { slot = 0; ph ^= 1u; }
                    // (a half batch's rows are loaded before the first is used: row by row a unit of 256 channels took 1634 clocks here
                    // and 2690 below, of 5800)
                    Eight<T> v[HALF];
#pragma unroll
                    for (int j = 0; j < HALF; ++j) read(v[j], base[h] + from[j]);
#pragma unroll
                    for (int j = 0; j < HALF; ++j) t[h * HALF + j] = v[j].part();
                }
                // The largest of each row over its lanes: lanes exchange halves of the sets until a lane has one set, then the rest.  Lane
                // j LPR / BATCH of a row's lanes ends with set j.  (A redux per row took 90 clocks each.)
#pragma unroll
                for (int n = BATCH / 2, o = LPR / 2; n > 0; n /= 2, o /= 2) {
                    const bool upper = sub & o;
#pragma unroll
                    for (int j = 0; j < n; ++j) {
                        const uint32_t keep = upper ? t[j + n] : t[j], give = upper ? t[j] : t[j + n];
                        t[j] = Eight<T>::of_two(keep, __shfl_xor_sync(0xffffffffu, give, o));
                    }
                }
#pragma unroll
                for (int o = LPR / BATCH / 2; o > 0; o /= 2) t[0] = Eight<T>::of_two(t[0], __shfl_xor_sync(0xffffffffu, t[0], o));
                const uint32_t mine = Eight<T>::whole(t[0]);
                if (!ok) break;
                const RowScale rs = row_scale(Eight<T>::top_f32(mine));
                if (batch == 0) {
                    ok = __all_sync(0xffffffffu, mbar_wait_parked(&ctl->a_empty[ab], (use & 1u) ^ 1u, abort_flag));
                    if (!ok) break;
                }
                if ((sub & (LPR / BATCH - 1)) == 0)
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(xs + (uint32_t)row_of(batch, sub / (LPR / BATCH)) * 4u), "f"(rs.scale) : "memory");
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (!there[h]) continue;
                    Eight<T> v[HALF];
                    float inv[HALF];
                    uint2 c[HALF];
#pragma unroll
                    for (int j = 0; j < HALF; ++j) read(v[j], base[h] + from[j]);
#pragma unroll
                    for (int j = 0; j < HALF; ++j) inv[j] = __shfl_sync(0xffffffffu, rs.inv, (lane & ~(LPR - 1)) + (h * HALF + j) * (LPR / BATCH));
#pragma unroll
                    for (int j = 0; j < HALF; ++j) c[j] = v[j].codes(inv[j]);
                    if (sub * 8 < g.kb * 128) {
                        const uint32_t rows_at = tile + (uint32_t)((2 * batch + h) * SLOT_ROWS) * 128u;
#pragma unroll
                        for (int j = 0; j < HALF; ++j)
                            asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(rows_at + to[j]), "r"(c[j].x), "r"(c[j].y) : "memory");
                    }
                    __syncwarp();                             // every lane has read this half
                    if (lane == 0) mbar_arrive(&ctl->rows_empty[qg][bar[h]]);
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
        uint64_t *add_bar = &ctl->add_full[ew];
        for (int c = (int)threadIdx.x - 64; c < (int)g.n_tiles * g.bn; c += 256) {
            scale_s[c] = c < g.n ? ws[c] : 0.f;
            shift_s[c] = c < g.n ? shift[c] : 0.f;
        }
        named_bar_sync(1, 256);
        const QuantOut<T> out{z, add, g.p, g.n, g.dense, g.relu};
        bool ok = true;
        uint32_t i = 0, s = 0, turn = 0, add_ph = 0;
        const bool boxed = g.dense && add;
        for (uint32_t u = blockIdx.x; ok && u < g.units; u += gridDim.x, ++i) {
            for (uint32_t nt = 0; ok && nt < g.n_tiles; ++nt, ++s) {
                if ((s & 1u) != egroup) continue;
                const uint32_t row0 = u * kQRows + quarter * 32, row = row0 + lane;
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
                ok = __all_sync(0xffffffffu, mbar_wait_parked(&ctl->xs_full[i % kQSlots], (i / kQSlots) & 1u, abort_flag));
                const float *xs = xs_s + (i % kQSlots) * kQRows + quarter * 32;
                f32x2 xs2[4];                    // 16-bit types: rows lane / 4 + 8 k, otherwise row `lane`
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float v1 = ok ? xs[g.dense && sizeof(T) == 2 ? lane / 4 + 8 * k : lane] : 0.f;
                    xs2[k] = pair(v1, v1);
                }
                ok = ok && __all_sync(0xffffffffu, mbar_wait_parked(&ctl->acc_full[s & 1u], (s >> 1) & 1u, abort_flag));
                if (!ok) {
                    if (boxed) { if (lane == 0) mbar_wait_parked(add_bar, add_ph, nullptr, 200000000ull); __syncwarp(); }
                    break;
                }
                tc_fence_after_sync();
                const uint32_t t_row = tmem_base + (s & 1u) * (uint32_t)g.bn + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
                for (int c0 = 0; c0 < cols; c0 += CH) {
                    uint8_t *buf = box();
                    if (boxed) {
                        ok = __all_sync(0xffffffffu, mbar_wait_parked(add_bar, add_ph, abort_flag));
                        if (!ok) {                              // (the copy in flight lands before the block ends)
                            if (lane == 0) mbar_wait_parked(add_bar, add_ph, nullptr, 200000000ull);
                            __syncwarp();
                            break;
                        }
                        add_ph ^= 1u;
                    }
                    quant_chunk<T, true>(out, buf, boxed, t_row + (uint32_t)c0, scale_s + n0 + c0, shift_s + n0 + c0, xs2, row, n0 + c0,
                                                    cols - c0, lane);
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
size_t fused_smem(const QuantFused &g, size_t slot) {
    const size_t w = (size_t)(g.resident ? (int)g.n_tiles * g.kb : g.stages) * g.bn * 128;
    return 1024 + 2 * (size_t)g.kb * kQBlock + w + (size_t)8 * g.nbuf * kQStage + (size_t)g.rings * g.depth * slot + 8 * (size_t)g.n_tiles * g.bn +
           kQSlots * kQRows * 4 + sizeof(QuantCtl) + 16;
}

}  // namespace

// Strides that leave pixels out; otherwise rows of X are side by side, whatever the strides.
static bool skips_pixels(const Problem &pb) { return pb.h_out != pb.h_in || pb.w_out != pb.w_in; }

// Rows enough for every SM, short ones that start on 16-byte boundaries, and not too many channels for two accumulators to drain.  This
// kernel and the two of quant_gemm.cu, us: 100352 rows 64 -> 256 18.8 and 25.9, 256 -> 64 19.5 and 28.1, 128 -> 128 14.7 and 22.4,
// 256 -> 1024 75.3 and 79.1, 64 -> 2048 143 and 123; 19200 rows 64 -> 256 7.8 and 9.6, 256 -> 64 8.3 and 8.7; below a unit per SM, 6272
// rows 256 -> 64, 7.2 and 6.1: a warp per row beats sixteen rows a warp.  256 channels are what 32 lanes read at once; an earlier form,
// slower by a fifth, that took longer rows in pieces was behind there (512 -> 1024 122.9 and 100.8; this form has not been tried).
bool quant_fused_eligible(const Problem &pb, int elem_bytes) {
    const bool beside = !skips_pixels(pb);                               // (otherwise im2col boxes of 64 channels)
    return pb.c_in <= 256 && pb.c_in % 8 == 0 && (size_t)pb.c_in * elem_bytes % 16 == 0 && pb.c_out <= 1024 &&
           (beside || (pb.c_in % 64 == 0 && pb.stride_h <= 8 && pb.stride_w <= 8)) && pb.p >= (long long)kQRows * device_sm_count();
}

RowMap quant_row_map(const Problem &pb) {
    RowMap r;
    r.step = pb.c_in;
    r.strided = skips_pixels(pb);
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
    g.strided = skips_pixels(pb);
    g.stride_h = pb.stride_h; g.stride_w = pb.stride_w;
    g.by_w = FastDiv((uint32_t)pb.w_out); g.by_h = FastDiv((uint32_t)pb.h_out);
    g.boxes = (pb.c_in * es + 127) / 128;
    g.p = (uint32_t)pb.p; g.k = pb.c_in; g.kb = (pb.c_in + 127) / 128; g.n = pb.c_out; g.relu = relu;
    g.dense = (size_t)pb.c_out * es % 16 == 0;
    g.units = (uint32_t)((pb.p + kQRows - 1) / kQRows);
    // Buffers.  Rows up to 128 elements: two boxes per epilogue warp and four slots of rows per group (64 -> 256 at 56 x 56, N = 128 55.5 us,
    // with one box and six slots 59.3); longer ones the other way round (256 -> 64, N = 256 107.3 and 111.5).  The weights resident,
    // otherwise at least three slots of them; wide tiles.
    const size_t room = 227 * 1024, set = 256 * es;
    g.rings = pb.c_in <= 64 ? 2 : 1;                                                         // (RowSets)
    const size_t warps = 8 / g.rings, sets = kQRows / warps / (pb.c_in <= 64 ? 4 : (pb.c_in <= 128 ? 2 : 1));
    const size_t slot = warps * (sets * set <= 4096 ? sets * set : 4096) / 2;
    const struct { int nbuf, depth; } wanted[] = {{pb.c_in <= 128 ? 2 : 1, pb.c_in <= 128 ? 4 : 6}, {1, 4}, {1, 3}, {1, 2}};
    size_t smem = 0;
    for (const auto &c : wanted) {
        g.nbuf = c.nbuf; g.depth = c.depth; g.stages = 3;
        for (int widest = 256; widest >= 64 && !smem; widest /= 2) {
            g.n_tiles = (uint32_t)((pb.c_out + widest - 1) / widest);
            g.bn = (int)(((pb.c_out + g.n_tiles - 1) / g.n_tiles + 63) / 64 * 64);
            for (g.resident = 1; g.resident >= 0; --g.resident)
                if ((smem = fused_smem(g, slot)) <= room) break;
                else smem = 0;
            if (smem) break;
        }
        if (smem) break;
    }
    if (!smem) return cudaErrorInvalidValue;
    while (g.rings == 1 && g.depth < kQMaxDepth) {                                           // the rest for longer rows
        ++g.depth;
        if (fused_smem(g, slot) > room) { --g.depth; break; }
    }
    smem = fused_smem(g, slot);
    const unsigned grid = g.units < (uint32_t)sms ? g.units : (unsigned)sms;
    CUtensorMap tx, tw, tz, ta;
    const int slot_rows = (int)(slot / (set / (pb.c_in <= 64 ? 4 : (pb.c_in <= 128 ? 2 : 1))));
    // (the box of base pixels has h_out x w_out positions: upper = (out - 1) stride - (in - 1))
    if (g.strided ? !make_tmap_im2col_bf16(&tx, x, pb.n, pb.h_in, pb.w_in, pb.c_in, 0, 0, (pb.h_out - 1) * pb.stride_h - (pb.h_in - 1),
                                           (pb.w_out - 1) * pb.stride_w - (pb.w_in - 1), pb.stride_h, pb.stride_w, slot_rows, 64)
                  : !make_tmap_matrix_bytes(&tx, x, pb.p, pb.c_in, es, slot_rows))
        return cudaErrorInvalidValue;
    if (!make_tmap_matrix_bytes(&tw, wq, pb.c_out, quant_pitch(pb), 1, g.bn)) return cudaErrorInvalidValue;
    tz = ta = tw;
    if (g.dense) {
        if (!make_tmap_matrix_bytes(&tz, z, pb.p, pb.c_out, es, 32)) return cudaErrorInvalidValue;
        if (add && !make_tmap_matrix_bytes(&ta, add, pb.p, pb.c_out, es, 32)) return cudaErrorInvalidValue;
    }
    int *err = nullptr;
    if (cudaError_t e = error_word_address(&err); e != cudaSuccess) return e;
    auto go = [&](auto tag, auto lpr) {
        using T = decltype(tag);
        auto kernel = quant_fused_kernel<T, decltype(lpr)::value>;
        static PerDevice attr, carve;
        if (cudaError_t e = max_dynamic_smem_once(kernel, 227 * 1024, &attr); e != cudaSuccess) return e;
        prefer_max_shared_once(kernel, &carve);
        return launch_pdl(kernel, dim3(grid), dim3(kQThreads), smem, st, tx, tw, tz, ta, g, ws, shift, (const T *)add, (T *)z, err);
    };
    auto typed = [&](auto tag) {
        using std::integral_constant;
        if (pb.c_in <= 64) return go(tag, integral_constant<int, 8>());
        if (pb.c_in <= 128) return go(tag, integral_constant<int, 16>());
        return go(tag, integral_constant<int, 32>());
    };
    return dtype == CONVBN_F32 ? typed(float()) : (dtype == CONVBN_F16 ? typed(__half()) : typed(__nv_bfloat16()));
}

}  // namespace convbn
