// Orthogonal updates of matrices whose shorter side is at most 128 (formulas, pairs of halves: ortho.cuh), in one launch without a round through
// memory: a cluster of blocks keeps X, each block `width` columns of it, and its own copy of A and P.
//
// What such a matrix costs is not its products (a step's are 2 us of one tensor core) but the ways between them.  On chip a product, its sums
// from tensor memory and the rounding to pairs follow one another with a barrier in between; only A, whose sums run over all columns, goes
// round the cluster: every block sends its part's rows to the block that adds them up, which hands the result to all.
// 64 x 64 in fp32 takes 19 us, 75 by the kernel for large matrices: a product is 1650 clocks, 950 from the first MMA's issue to the last one's
// end and 650 for sums and rounding, the way in 2 us, out 1.  128 x 1152 takes 79 us: 9000 of a step's 25000 clocks are A's round, 128 KB into each block
// at about the rate of distributed shared memory.
// X lies as m rows x n columns whichever side is the shorter: a tall matrix is transposed on its way in and out.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "ortho.cuh"
#include "sm100_ptx.cuh"

namespace convbn {

using namespace ptx;

namespace {

constexpr int kSThreads = 512;                          // sixteen warps: a row of sums is four threads' work
constexpr uint32_t kSTile = 2 * kOrthoTile;            // 128 rows x 64 columns, hi and lo
constexpr int kSMaxWidth = 256;
constexpr int kSMaxCluster = 16;                       // (more than eight where the device has room for such a cluster)

struct SmallCtl {
    uint64_t done, rows;                               // a product; the other blocks' rows of A
    double sum, part[kSThreads / 32];
    uint32_t tmem_base;
};

// A launch's matrices: one cluster each.
struct SmallShape {
    int blocks, width;                                 // of a cluster; columns of a block (a multiple of 64)
};

__device__ __forceinline__ void st_cluster_v4(uint32_t addr, uint4 v) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ double ld_cluster_f64(uint32_t addr) {
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
    return v;
}
// (of all memory it takes 700 clocks, a fifth of a product)
__device__ __forceinline__ void fence_proxy_async_cluster() { asm volatile("fence.proxy.async.shared::cluster;" ::: "memory"); }

// To another block of the cluster; its barrier counts the bytes.
__device__ __forceinline__ void bulk_send(uint32_t dst, uint32_t src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "r"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// Eight numbers (2^10 times what they stand for) as pairs of halves.
__device__ __forceinline__ void to_pairs(const float (&v)[8], uint4 &hi, uint4 &lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const __half2 a = __floats2half2_rn(v[2 * e], v[2 * e + 1]);
        const float2 back = __half22float2(a);
        const __half2 b = __floats2half2_rn(v[2 * e] - back.x, v[2 * e + 1] - back.y);
        h[e] = *reinterpret_cast<const uint32_t *>(&a);
        l[e] = *reinterpret_cast<const uint32_t *>(&b);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}
// Eight numbers as they are, each in two words of 16 bits.
__device__ __forceinline__ void split_words(const float (&v)[8], uint4 &hi, uint4 &lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t a = __float_as_uint(v[2 * e]), b = __float_as_uint(v[2 * e + 1]);
        h[e] = a >> 16 | (b & 0xFFFF0000u);
        l[e] = (a & 0xFFFFu) | b << 16;
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ float2 from_pair(uint32_t hi, uint32_t lo) {
    const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&hi)), l = __half22float2(*reinterpret_cast<const __half2 *>(&lo));
    return make_float2(h.x + l.x, h.y + l.y);
}
__device__ __forceinline__ void from_pairs(uint4 hi, uint4 lo, float (&v)[8]) {
    const float2 a = from_pair(hi.x, lo.x), b = from_pair(hi.y, lo.y), c = from_pair(hi.z, lo.z), d = from_pair(hi.w, lo.w);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
}

template <class U, int V>
struct alignas(V * sizeof(U)) Few { U e[V]; };
template <int V, class U>
__device__ __forceinline__ Few<U, V> load(const U *p) { return *(const Few<U, V> *)p; }

template <class T>
__global__ void __launch_bounds__(kSThreads, 1) ortho_small_kernel(const __grid_constant__ OrthoTable tab, const SmallShape sh, int *err) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *x = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);          // [width / 64] tiles
    uint8_t *ap = x + (size_t)(sh.width / 64) * kSTile;                                // two tiles: A, then P; parts of A's sums before
    SmallCtl *ctl = (SmallCtl *)(ap + 2 * kSTile);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3, fourth = warp >> 2;
    const int blocks = sh.blocks, rank = blocks > 1 ? (int)cluster_rank() : 0;
    const int matrix = blockIdx.x / blocks;
    int which = 0;
    while (which + 1 < tab.items && tab.item[which + 1].first_matrix <= matrix) ++which;
    const OrthoItem &it = tab.item[which];
    const bool tall = it.rows > it.cols;
    const int m = min(it.rows, it.cols), n = max(it.rows, it.cols);
    const int col0 = rank * sh.width, cols = max(0, min(sh.width, n - col0));          // this block's columns
    const int m16 = (m + 15) & ~15, n16 = (cols + 15) & ~15, tiles = (cols + 63) / 64;
    const long long base = (long long)(matrix - it.first_matrix) * it.rows * it.cols;
    if (threadIdx.x == 0) {
        mbar_init(&ctl->done, 1);
        mbar_init(&ctl->rows, 1);
        fence_barrier_init();
    }
    if (warp == 0) {
        tmem_alloc(&ctl->tmem_base, 512);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (blocks > 1) cluster_sync_all();
    pdl_wait();
    pdl_launch_dependents();
    const uint32_t tmem = ctl->tmem_base;

    // ---- X = G / (|G| + eps); muon: the momentum's step on the way ----
    // (the block's tiles: zeros beyond the matrix)
    for (int i = threadIdx.x; i < tiles * (int)(kSTile / 16); i += kSThreads) ((uint4 *)x)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    // The block's elements in the order of memory, a thread one to four side by side of every kSThreads', sixteen in all under way; f(where a unit lies
    // in memory, and in the tiles, how many are there).  Four where a line's length and all addresses allow: 64 x 64 took 3700 clocks one by one.
    const int fast = tall ? m : cols, lines = tall ? cols : m, start = tall ? col0 * it.cols : col0;
    auto in_order = [&](auto side, auto &&f) {
        constexpr int V = decltype(side)::value, B = 16 / V;
        const int units = max(fast / V, 1), total = lines * (fast / V), dl = kSThreads / units, da = kSThreads - dl * units;
        int line = threadIdx.x / units, a = threadIdx.x - line * units;
        for (int e = threadIdx.x; e < total; e += B * kSThreads) {
            int at[B];
            uint32_t where[B];
#pragma unroll
            for (int k = 0; k < B; ++k) {
                const int i = tall ? a * V : line, j = tall ? line : a * V;
                at[k] = start + line * it.cols + a * V;
                where[k] = (j >> 6) * kSTile + ortho_chunk(i, (j & 63) >> 3) + (j & 7) * 2;
                line += dl;
                a += da;
                if (a >= units) { a -= units; ++line; }
            }
            f(at, where, (total - e + kSThreads - 1) / kSThreads);
        }
    };
    // a unit lies along a row of a tile or, tall, down its rows (the first a multiple of V): the q-th's place
    auto down = [&](uint32_t where, int q) { return (where + q * 128u) ^ (uint32_t)(q << 4); };
    const bool fours = it.cols % 4 == 0 && ((uintptr_t)it.g | (uintptr_t)it.momentum | (uintptr_t)it.master) % 16 == 0 && (uintptr_t)it.out % (4 * sizeof(T)) == 0;
    double s = 0.;
    // Once from memory: the sum of squares, and the number's two halves where hi and lo of it will be.
    // (Line by line, and again for the scaling, this took two thirds of 189 x 37's 70 us.)
    auto take = [&](auto side) {
        constexpr int V = decltype(side)::value, B = 16 / V;
        in_order(side, [&](const int (&at)[B], const uint32_t (&where)[B], int here) {
            float u[B][V];
            if (tab.muon) {
                Few<float, V> g[B], v[B];
#pragma unroll
                for (int k = 0; k < B; ++k)
                    if (k < here) { g[k] = load<V>((const float *)it.g + base + at[k]); v[k] = load<V>(it.momentum + base + at[k]); }
#pragma unroll
                for (int k = 0; k < B; ++k) {
                    if (k >= here) break;
#pragma unroll
                    for (int q = 0; q < V; ++q) {
                        v[k].e[q] = fmaf(tab.momentum, v[k].e[q], g[k].e[q]);
                        u[k][q] = tab.nesterov ? fmaf(tab.momentum, v[k].e[q], g[k].e[q]) : v[k].e[q];
                    }
                    *(Few<float, V> *)(it.momentum + base + at[k]) = v[k];
                }
            } else {
                Few<T, V> g[B];
#pragma unroll
                for (int k = 0; k < B; ++k)
                    if (k < here) g[k] = load<V>((const T *)it.g + base + at[k]);
#pragma unroll
                for (int k = 0; k < B; ++k)
#pragma unroll
                    for (int q = 0; q < V; ++q)
                        if (k < here) u[k][q] = to_f32(g[k].e[q]);
            }
#pragma unroll
            for (int k = 0; k < B; ++k) {
                if (k >= here) break;
                Few<uint16_t, V> h, l;
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    s += (double)u[k][q] * (double)u[k][q];
                    const uint32_t bits = __float_as_uint(u[k][q]);
                    h.e[q] = (uint16_t)(bits >> 16);
                    l.e[q] = (uint16_t)bits;
                }
                if (!tall) {
                    *(Few<uint16_t, V> *)(x + where[k]) = h;
                    *(Few<uint16_t, V> *)(x + where[k] + kOrthoTile) = l;
                    continue;
                }
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    uint8_t *to = x + down(where[k], q);
                    *(uint16_t *)to = h.e[q];
                    *(uint16_t *)(to + kOrthoTile) = l.e[q];
                }
            }
        });
    };
    if (fours) take(std::integral_constant<int, 4>()); else take(std::integral_constant<int, 1>());
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) ctl->part[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = ctl->part[0];
        for (int i = 1; i < kSThreads / 32; ++i) s += ctl->part[i];
        ctl->sum = s;
    }
    if (blocks > 1) cluster_sync_all(); else __syncthreads();
    s = 0.;
    if (blocks > 1) for (int b = 0; b < blocks; ++b) s += ld_cluster_f64(cluster_addr(&ctl->sum, b));
    else s = ctl->sum;
    const OrthoScaling scaled = OrthoScaling::of(s, tab.eps);
    // (rows beyond the matrix are zeros)
    for (int c = threadIdx.x; c < tiles * m16 * 8; c += kSThreads) {
        uint8_t *to = x + (size_t)(c / (m16 * 8)) * kSTile + c % (m16 * 8) * 16;
        const uint4 top = *(const uint4 *)to, low = *(const uint4 *)(to + kOrthoTile);
        const uint32_t a[4] = {top.x, top.y, top.z, top.w}, b[4] = {low.x, low.y, low.z, low.w};
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = scaled(__uint_as_float(a[e] << 16 | (b[e] & 0xFFFFu)));
            v[2 * e + 1] = scaled(__uint_as_float((a[e] & 0xFFFF0000u) | b[e] >> 16));
        }
        uint4 h, l;
        to_pairs(v, h, l);
        *(uint4 *)to = h;
        *(uint4 *)(to + kOrthoTile) = l;
    }

    uint32_t ph = 0;
    const uint32_t x_at = smem_u32(x), ap_at = smem_u32(ap), hi_word = smem_desc_hi_sw128(1024);
    // d (+ 256: the products with a lo) = A-operand x B-operand over k steps of 16; tiles of 64 k or 64 n are kSTile apart
    // (wide: operands, or what the sums will lie on, are other blocks' doing)
    auto product = [&](uint32_t a_at, uint32_t b_at, bool b_mn, int nn, int steps, bool wide) {
        if (wide) {
            fence_proxy_async_cluster();
            cluster_sync_all();
        } else {
            fence_proxy_async_smem();
            __syncthreads();
        }
        if (warp == 0 && steps > 0 && elect_one()) {
            tc_fence_after_sync();
            if (wide) fence_proxy_async_cluster();
            const uint32_t idesc = idesc_h16_f32(128, nn, 0, b_mn, 1);
            for (int k = 0; k < steps; ++k) {
                const uint32_t a = smem_desc_lo(a_at + (k >> 2) * kSTile, 16) + (k & 3) * 2u;
                const uint32_t b = b_mn ? smem_desc_lo(b_at, kSTile) + k * 128u : smem_desc_lo(b_at + (k >> 2) * kSTile, 16) + (k & 3) * 2u;
                umma_bf16_ss_sel(tmem, a, hi_word, b, hi_word, idesc, k);
                umma_bf16_ss_sel(tmem + 256, a, hi_word, b + (kOrthoTile >> 4), hi_word, idesc, k);
                umma_bf16_ss_halves<true>(tmem + 256, a + (kOrthoTile >> 4), hi_word, b, hi_word, idesc);
            }
            umma_commit(&ctl->done);
        }
    };
    auto finished = [&](int steps) {
        if (steps > 0) {
            if (!mbar_wait_bounded(&ctl->done, ph, nullptr) && threadIdx.x == 0) atomicOr(err, ERRW_TIMEOUT);
            ph ^= 1u;
        }
        tc_fence_after_sync();
    };
    const uint32_t row = quarter * 32 + lane, t_row = tmem + ((uint32_t)(quarter * 32) << 16);
    // 16 sums of this thread's row from column c on, times f
    auto sums = [&](int c, float f, float (&v)[16]) {
        uint32_t p[16], q[16];
        tmem_ld_32x16(t_row + c, p);
        tmem_ld_32x16(t_row + 256 + c, q);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = f * (__uint_as_float(p[i]) + __uint_as_float(q[i]));
    };
    auto chunk_of = [&](uint8_t *at, int c) { return at + (size_t)(c >> 6) * kSTile + ortho_chunk(row, (c & 63) >> 3); };
    // sixteen numbers of a row from column c on
    auto read = [&](uint8_t *at, int c, float (&v)[16]) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint8_t *from = chunk_of(at, c + 8 * q);
            float w[8];
            from_pairs(*(const uint4 *)from, *(const uint4 *)(from + kOrthoTile), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[8 * q + e] = w[e];
        }
    };
    auto write = [&](uint8_t *at, int c, const float (&v)[16], bool whole) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint8_t *to = chunk_of(at, c + 8 * q);
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = v[8 * q + e];
            uint4 h, l;
            if (whole) split_words(w, h, l); else to_pairs(w, h, l);
            *(uint4 *)to = h;
            *(uint4 *)(to + kOrthoTile) = l;
        }
    };
    const bool rows_here = quarter * 32 < m16;                        // (whole warps)

    for (int step = 0; step < tab.steps; ++step) {
        // ---- A = X X^T ----
        product(x_at, x_at, false, m16, n16 / 16, blocks > 1);
        finished(n16 / 16);
        float v[16], old[16];
        if (blocks == 1) {
            if (rows_here)
                for (int c = fourth * 16; c < m16; c += 64) {
                    sums(c, 1.f / kOrthoScale, v);
                    write(ap, c, v, false);
                }
        } else {
            // part by part to the block that has the row: [block][4 columns][its rows] in fp32, where P was (rows side by side, as a warp has
            // them: with a row's columns side by side the sums' round took 7 us)
            const int share = 128 / blocks;                           // (blocks: a power of two, 16 at most)
            if (rows_here) {
                const uint32_t to = cluster_addr(ap, row / share) + (rank * 32 * share + row % share) * 16;
                for (int c = fourth * 16; c < m16; c += 64) {
                    if (n16 > 0) sums(c, 1.f, v);
                    else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = 0.f;
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        st_cluster_v4(to + (c / 4 + q) * share * 16, make_uint4(__float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]),
                                                                     __float_as_uint(v[4 * q + 3])));
                }
            }
            tc_fence_before_sync();
            cluster_sync_all();
            // each thread eight columns of a row of the share, in turn
            constexpr int kSets = 128 / 2 * 16 / kSThreads;           // of two blocks: their shares are the largest
            float w[kSets][8];
#pragma unroll
            for (int k = 0; k < kSets; ++k) {
                const int idx = threadIdx.x + k * kSThreads, r = idx % share, c = idx / share * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[k][e] = 0.f;
                if (c < m16)
                    for (int b = 0; b < blocks; ++b) {
                        const float4 *f = (const float4 *)ap + (b * 32 + c / 4) * share + r;
                        const float4 f0 = f[0], f1 = f[share];
                        w[k][0] += f0.x; w[k][1] += f0.y; w[k][2] += f0.z; w[k][3] += f0.w;
                        w[k][4] += f1.x; w[k][5] += f1.y; w[k][6] += f1.z; w[k][7] += f1.w;
                    }
            }
            fence_proxy_async_cluster();
            cluster_sync_all();
#pragma unroll
            for (int k = 0; k < kSets; ++k) {
                const int idx = threadIdx.x + k * kSThreads, r = rank * share + idx % share, c = idx / share * 8;
                if (c >= m16 || r >= m16) continue;
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = w[k][e] * (1.f / kOrthoScale);
                uint4 h, l;
                to_pairs(f, h, l);
                uint8_t *to = ap + (uint32_t)(c >> 6) * kSTile + ortho_chunk(r, (c & 63) >> 3);
                *(uint4 *)to = h;
                *(uint4 *)(to + kOrthoTile) = l;
            }
            // its rows, side by side in each tile, to every other block by bulk copies (by the threads' stores of 16 bytes, a line each, the
            // round took 9400 clocks of 128 x 1152's 34000 a step)
            fence_proxy_async_smem();
            __syncthreads();
            const int mine = max(0, min(share, m16 - rank * share)), parts = 2 * ((m16 + 63) / 64);
            if (threadIdx.x == 0 && m16 > mine) mbar_arrive_expect_tx(&ctl->rows, (m16 - mine) * 128 * parts);
            if (mine > 0)
                for (int i = threadIdx.x; i < blocks * parts; i += kSThreads) {
                    const int to = i / parts, part = i - to * parts;
                    if (to == rank) continue;
                    uint8_t *from = ap + part * kOrthoTile + rank * share * 128;
                    bulk_send(cluster_addr(from, to), smem_u32(from), mine * 128, cluster_addr(&ctl->rows, to));
                }
            if (m16 > mine) {
                if (!mbar_wait_bounded(&ctl->rows, step & 1, nullptr) && threadIdx.x == 0) atomicOr(err, ERRW_TIMEOUT);
            }
            // (A's rows have come: said to the blocks they came from, which read them until then and write P over them below)
            __syncwarp();
            cluster_arrive_all();
        }
        tc_fence_before_sync();
        // ---- P = b A + c A A, where A is ----
        // (the first of a thread's old numbers are read while the tensor core works)
        const int c0 = fourth * 16;
        product(ap_at, ap_at, false, m16, m16 / 16, false);
        if (rows_here && c0 < m16) read(ap, c0, old);
        finished(m16 / 16);
        if (blocks > 1) {
            __syncwarp();
            cluster_wait_all();
        }
        if (rows_here)
            for (int c = c0; c < m16; c += 64) {
                if (c != c0) read(ap, c, old);
                sums(c, kOrthoCoefC / kOrthoScale, v);
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = fmaf(kOrthoCoefB, old[e], v[e]);
                write(ap, c, v, false);
            }
        tc_fence_before_sync();
        // ---- X <- a X + P X, in place (rows and columns beyond the matrix stay zero) ----
        product(ap_at, x_at, true, n16, n16 > 0 ? m16 / 16 : 0, false);
        if (rows_here && c0 < n16) read(x, c0, old);
        finished(n16);
        const bool last = step + 1 == tab.steps;
        if (rows_here)
            for (int c = c0; c < n16; c += 64) {
                if (c != c0) read(x, c, old);
                sums(c, 1.f / kOrthoScale, v);
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = (int)row < m ? fmaf(kOrthoCoefA, old[e], v[e]) : 0.f;
                write(x, c, v, last);
            }
        tc_fence_before_sync();
    }
    __syncthreads();
    // ---- out, in the order of memory ----
    auto give = [&](auto side) {
        constexpr int V = decltype(side)::value, B = 16 / V;
        in_order(side, [&](const int (&at)[B], const uint32_t (&where)[B], int here) {
            Few<float, V> o[B], old[B];
            if (tab.muon)
#pragma unroll
                for (int k = 0; k < B; ++k)
                    if (k < here) old[k] = load<V>(it.master + base + at[k]);
#pragma unroll
            for (int k = 0; k < B; ++k)
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    if (k >= here) continue;
                    const uint8_t *from = x + (tall ? down(where[k], q) : where[k] + q * 2u);
                    o[k].e[q] = __uint_as_float((uint32_t)*(const uint16_t *)from << 16 | *(const uint16_t *)(from + kOrthoTile)) * (1.f / kOrthoScale);
                }
#pragma unroll
            for (int k = 0; k < B; ++k) {
                if (k >= here) break;
                if (tab.muon) {
#pragma unroll
                    for (int q = 0; q < V; ++q) o[k].e[q] = fmaf(-it.scale, o[k].e[q], tab.keep * old[k].e[q]);
                    *(Few<float, V> *)(it.master + base + at[k]) = o[k];
                }
                if (it.out) {
                    Few<T, V> r;
#pragma unroll
                    for (int q = 0; q < V; ++q) r.e[q] = from_f32<T>(o[k].e[q]);
                    *(Few<T, V> *)((T *)it.out + base + at[k]) = r;
                }
            }
        });
    };
    if (fours) give(std::integral_constant<int, 4>()); else give(std::integral_constant<int, 1>());
    __syncthreads();
    if (blocks > 1) cluster_sync_all();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

// One shape for all of a launch's matrices: as wide as the longest needs.
bool small_shape(const OrthoTable &t, SmallShape *s) {
    int longest = 0;
    for (int i = 0; i < t.items; ++i) {
        const int m = std::min(t.item[i].rows, t.item[i].cols), n = std::max(t.item[i].rows, t.item[i].cols);
        if (m > 128 || n > kSMaxCluster * kSMaxWidth) return false;
        longest = std::max(longest, n);
    }
    s->blocks = 1;
    // (few wide blocks: 66 x 150 by two blocks of 128 columns took twice as long as by one)
    while (longest > s->blocks * kSMaxWidth) s->blocks *= 2;
    s->width = ((longest + s->blocks - 1) / s->blocks + 63) / 64 * 64;
    return true;
}

template <class T>
cudaLaunchConfig_t small_config(const OrthoTable &t, const SmallShape &s, cudaLaunchAttribute (&at)[2]) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(t.matrices * s.blocks));
    cfg.blockDim = dim3(kSThreads);
    // The whole shared memory whatever the width: blocks of two clusters on one SM could each hold the tensor memory that the other cluster
    // waits for.
    cfg.dynamicSmemBytes = 1024 + (kSMaxWidth / 64 + 2) * kSTile + sizeof(SmallCtl);
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = s.blocks;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = s.blocks > 1 ? 2 : 1;
    return cfg;
}
template <class T>
cudaError_t small_attributes() {
    static PerDevice smem, wide;
    auto kernel = ortho_small_kernel<T>;
    if (cudaError_t e = max_dynamic_smem_once(kernel, 1024 + (kSMaxWidth / 64 + 2) * (int)kSTile + (int)sizeof(SmallCtl), &smem); e != cudaSuccess) return e;
    bool &done = wide.done[current_device_slot()];
    if (done) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) done = true;
    return e;
}
// Whether the device holds such clusters (of sixteen blocks not every one does), and this is the shorter way.  A B200 runs 7 clusters of sixteen blocks at
// a time, 15 of eight, 33 of four, 74 of two; the next ones are another round, where the kernel for large matrices fills the SMs and its chain of
// waits is paid once.  Estimates in us, five steps.  Measured, this kernel and the other, fp32: one 16 x 2268 58 and 136, one 128 x 4096 116 and 148; eight of those
// 216 and 170; 128 x 2048 by 8 108 and 145, by 16 206 and 160; 64 x 64 by 512 89 and 306.
template <class T>
bool small_pays(const OrthoTable &t, const SmallShape &s) {
    static std::atomic<int> known[kMaxDevices][5];     // clusters at a time + 1 (threads that ask at once find the same)
    int log = 0;
    while (1 << log < s.blocks) ++log;
    std::atomic<int> &answer = known[current_device_slot()][log];
    int fit = answer.load(std::memory_order_relaxed) - 1;
    if (fit < 0) {
        if (s.blocks == 1) {
            fit = device_sm_count();
        } else {
            cudaLaunchAttribute at[2];
            const cudaLaunchConfig_t cfg = small_config<T>(t, s, at);
            if (small_attributes<T>() != cudaSuccess || cudaOccupancyMaxActiveClusters(&fit, ortho_small_kernel<T>, &cfg) != cudaSuccess) {
                cudaGetLastError();
                fit = 0;
            }
        }
        answer.store(fit + 1, std::memory_order_relaxed);
    }
    if (fit < 1) return false;
    int side = 0;
    float other = 110.f;
    for (int i = 0; i < t.items; ++i) {
        const OrthoItem &it = t.item[i];
        side = std::max(side, std::min(it.rows, it.cols));
        other += (it.wide ? 0.037f : 0.06f) * (float)(3 * std::max(it.rt, it.ct) + 1) * (float)it.count;
    }
    const float round = 10.f + (float)side * (0.15f + 0.001f * (float)s.width) + (s.blocks > 1 ? 30.f : 0.f);
    return t.matrices <= fit || round * (float)((t.matrices + fit - 1) / fit) <= other;
}

template <class T>
cudaError_t launch_small_t(const OrthoTable &t, const SmallShape &s, cudaStream_t st) {
    int *err = nullptr;
    if (cudaError_t e = error_word_address(&err); e != cudaSuccess) return e;
    if (cudaError_t e = small_attributes<T>(); e != cudaSuccess) return e;
    cudaLaunchAttribute at[2];
    cudaLaunchConfig_t cfg = small_config<T>(t, s, at);
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, ortho_small_kernel<T>, t, s, err);
}

}  // namespace

bool ortho_small_pays(const OrthoTable &t) {
    SmallShape s;
    if (!small_shape(t, &s)) return false;
    switch (t.dtype) {
        case CONVBN_F32: return small_pays<float>(t, s);
        case CONVBN_F16: return small_pays<__half>(t, s);
        default: return small_pays<__nv_bfloat16>(t, s);
    }
}

cudaError_t launch_ortho_small(const OrthoTable &t, cudaStream_t st) {
    SmallShape s;
    if (!small_shape(t, &s)) return cudaErrorInvalidValue;
    switch (t.dtype) {
        case CONVBN_F32: return launch_small_t<float>(t, s, st);
        case CONVBN_F16: return launch_small_t<__half>(t, s, st);
        default: return launch_small_t<__nv_bfloat16>(t, s, st);
    }
}

}  // namespace convbn
