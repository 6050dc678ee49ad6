// Group norm with its activation over channels-last activations, forward and backward (formulas: group_norm.cuh).
//
// A block takes a slab of channels (whole groups, 128 bytes of a pixel or more, so that every access of a warp is whole lines) and a run of
// pixels of one sample; a thread keeps its channels, so what belongs to a channel stays in registers.
//   on chip     where one block holds the slab of a sample in shared memory (or a cluster does, where there are few slabs): read once.
//   two passes  otherwise: the first sums, the second reads the same tensors again, the latest first, from L2 as far as that has them, and
//               writes.
// Bound by memory; what is lost are the ends of passes, where sums go round.  So a run is long, its sums are shared by warp shuffles first,
// and few runs are left for the second pass to join: clusters of eight blocks join theirs.
// Measured, against each tensor once at the rate of a copy: forward 32 x 56 x 56 x 256 bf16 30.4 us (15.7; two plain passes, read and copied, take 27 to 31),
// 2 x 200 x 334 x 256 43.7 (20.8), 64 x 112 x 112 x 96 half with SiLU 97 (47); backward 64 x 7 x 7 x 2048 on chip 18 to 20 (5.9), 2 x 200 x 334 x 256
// 61 (31), 64 x 112 x 112 x 96 150 (70).  On chip the first took 27 in an early form of the kernel and 39 to 44 in a later one.
#include "group_norm.cuh"

#include <algorithm>

#include "sm100_ptx.cuh"

namespace convbn {

namespace {

constexpr int kThreads = 256;                  // of the two passes' blocks
constexpr int kKept = 224;                     // bytes of shared memory that a thread keeps pixels in: 1024 threads' share is the SM's
constexpr int kMaxKeptThreads = 512;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int V>
__device__ __forceinline__ float at(const f32x2 (&v)[(V + 1) / 2], int i) {
    const float2 f = split2(v[i / 2]);
    return i % 2 ? f.y : f.x;
}
// Sums over a warp's rows of threads, where tx divides 32 (lanes below tx have them).
__device__ __forceinline__ float fold(const GroupNormShape &s, float v) {
    if (s.fold)
        for (int o = s.tx; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Where a thread's sums go in a block's table [rows][tx]: rows are warps after fold(), else rows of threads; -1: nowhere.
__device__ __forceinline__ int table_row(const GroupNormShape &s) {
    const int lane = threadIdx.x & 31;
    if (s.fold) return lane < s.tx ? (int)threadIdx.x >> 5 : -1;
    const int ty = threadIdx.x / s.tx;
    return ty < s.ty ? ty : -1;
}
__device__ __forceinline__ int table_rows(const GroupNormShape &s) { return s.fold ? (int)blockDim.x >> 5 : s.ty; }
// Sums of `red`, [rows][width], over its rows (they end up in the first) and over groups of `size` neighbours: out(group, sum).
template <class F>
__device__ __forceinline__ void group_sums(float *red, int rows, int width, int size, int groups, F &&out) {
    if (rows > 1 && size > 1) {
        for (int c = threadIdx.x; c < width; c += blockDim.x) {
            float v = red[c];
            for (int r = 1; r < rows; ++r) v += red[r * width + c];
            red[c] = v;
        }
        rows = 1;
        __syncthreads();
    }
    if (size <= 16) {                                           // a thread per group
        for (int g = threadIdx.x; g < groups; g += blockDim.x) {
            float v = 0.f;
            for (int r = 0; r < rows; ++r)
                for (int i = 0; i < size; ++i) v += red[r * width + g * size + i];
            out(g, v);
        }
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int g = warp; g < groups; g += blockDim.x >> 5) {
        float v = 0.f;
        for (int i = lane; i < size; i += 32) v += red[g * size + i];
        v = warp_sum(v);
        if (lane == 0) out(g, v);
    }
}

// Element g of the table `own` of each block of a cluster of `blocks`; all loads are on their way before the first is waited for (one after the
// other they took 4 us of a pass).
constexpr int kMaxCluster = 8;
__device__ __forceinline__ void cluster_pairs(const float2 *own, int blocks, float2 (&v)[kMaxCluster]) {
    uint32_t at[kMaxCluster];
#pragma unroll
    for (int b = 0; b < kMaxCluster; ++b) at[b] = ptx::cluster_addr(own, b < blocks ? b : 0);
#pragma unroll
    for (int b = 0; b < kMaxCluster; ++b) asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v[b].x), "=f"(v[b].y) : "r"(at[b]) : "memory");
}
// Means and squared distances of the blocks' runs, joined: run b has weight(b) values a channel (none: zero).
template <class W>
__device__ __forceinline__ float2 join_runs(const float2 *own, int blocks, float total, float cg, W &&weight) {
    float2 v[kMaxCluster];
    cluster_pairs(own, blocks, v);
    float m = 0.f, q = 0.f;
#pragma unroll
    for (int b = 0; b < kMaxCluster; ++b)
        if (b < blocks) m = fmaf(weight(b) / total, v[b].x, m);
#pragma unroll
    for (int b = 0; b < kMaxCluster; ++b)
        if (b < blocks) {
            const float d = v[b].x - m;
            q += fmaf(weight(b) * cg * d, d, v[b].y);
        }
    return make_float2(m, q);
}

// minus_mean, scale, beta of the V channels from c0 on (c0 and stat: within the slab); what lies beside V = 1's channel is zero.
template <int V, bool ONE, class F>
__device__ __forceinline__ void set_channels(NormChannels<V, ONE> &k, int c0, int cg, const float *gamma, const float *beta, F &&stat) {
    float2 one;
    if constexpr (ONE) one = stat(c0 / cg);
#pragma unroll
    for (int i = 0; i < NormChannels<V, ONE>::P; ++i) {
        float m[2] = {0.f, 0.f}, sc[2] = {0.f, 0.f}, b[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < (V > 1 ? 2 : 1); ++e) {
            const int c = c0 + 2 * i + e;
            const float2 st = ONE ? one : stat(c / cg);
            m[e] = -st.x;
            sc[e] = __ldg(gamma + c) * st.y;
            b[e] = __ldg(beta + c);
        }
        if (!ONE || i == 0) k.minus_mean[ONE ? 0 : i] = pair(m[0], m[1]);
        k.scale[i] = pair(sc[0], sc[1]);
        k.beta[i] = pair(b[0], b[1]);
    }
}
template <int V, bool ONE>
__device__ __forceinline__ float near_zero(const NormChannels<V, ONE> &k) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) top = fmaxf(top, fabsf(at<V>(k.beta, i)));
    return top * 0x1p-20f;
}

// ---- sums of a run ------------------------------------------------------------------------------------------------------------------------
// A thread's values as distances from its channel's first one, which is one of the values: what the sums lose by rounding is small against the
// spread that the value itself brings in, however far the mean is from zero.
template <class T, int V>
struct Spread {
    static constexpr int P = (V + 1) / 2;
    f32x2 ck[P], cs[P], cq[P];                       // per channel: minus the first value, sums of distances and of their squares
    __device__ __forceinline__ void none() {
#pragma unroll
        for (int i = 0; i < P; ++i) ck[i] = cs[i] = cq[i] = 0ull;
    }
    __device__ __forceinline__ void first(const NormVec<T, V> &v) {
#pragma unroll
        for (int i = 0; i < P; ++i) { ck[i] = mul2(v.get(i), both(-1.f)); cs[i] = cq[i] = 0ull; }
    }
    __device__ __forceinline__ void add(const NormVec<T, V> &v) {
#pragma unroll
        for (int i = 0; i < P; ++i) { const f32x2 d = add2(v.get(i), ck[i]); cs[i] = add2(cs[i], d); cq[i] = fma2(d, d, cq[i]); }
    }
    __device__ __forceinline__ float mean(int i, float inv) const { return fmaf(at<V>(cs, i), inv, -at<V>(ck, i)); }
    // squared distances from m
    __device__ __forceinline__ float square(int i, float k, float inv, float m) const {
        const float c = at<V>(cs, i), d = fmaf(c, inv, -at<V>(ck, i)) - m;
        return fmaf(-c * inv, c, at<V>(cq, i)) + k * d * d;
    }
};
// Of a thread's columns, where they belong to one group: count, mean, squared distances (Chan, Golub, LeVeque: pairwise updates of a variance).
struct Moments {
    float cnt = 0.f, mean = 0.f, m2 = 0.f;
    template <class T, int V>
    __device__ __forceinline__ void join(const Spread<T, V> &p, int seen) {
        const float k = (float)seen, inv = 1.f / k;
        float m = 0.f, q = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) m += p.mean(i, inv);
        m *= 1.f / V;
#pragma unroll
        for (int i = 0; i < V; ++i) q += p.square(i, k, inv, m);
        const float add = k * V, all = cnt + add, d = m - mean, share = add / all;
        mean = fmaf(d, share, mean);
        m2 += q + d * d * (cnt * share);
        cnt = all;
    }
};
// The block's groups: out(group, (mean, squared distances)).  `one`: m holds the thread's values, else p does, `seen` of each channel.
template <class T, int V, class F>
__device__ __forceinline__ void block_moments(const GroupNormShape &s, float *red, float *mu, bool one, const Moments &m, const Spread<T, V> &p, int seen,
                                              float rows, F &&out) {
    const int tx = threadIdx.x % s.tx, to = table_row(s), lines = table_rows(s);
    const float total = 1.f / (rows * (float)s.cg);
    if (one) {
        // threads' columns of a group are neighbours
        const int per = s.slab_g == 1 ? s.tx : s.cg / V, g = s.slab_g == 1 ? 0 : tx / per;
        const float a = fold(s, m.cnt * m.mean);
        if (to >= 0) red[to * s.tx + tx] = a;
        __syncthreads();
        group_sums(red, lines, s.tx, per, s.slab_g, [&](int k, float v) { mu[k] = v * total; });
        __syncthreads();
        const float d = m.mean - mu[g], b = fold(s, m.cnt > 0.f ? m.m2 + m.cnt * d * d : 0.f);
        if (to >= 0) red[to * s.tx + tx] = b;
        __syncthreads();
        group_sums(red, lines, s.tx, per, s.slab_g, [&](int k, float v) { out(k, make_float2(mu[k], v)); });
    } else {
        const float k = (float)seen, inv = seen ? 1.f / k : 0.f;
        const int width = s.tx * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float a = fold(s, k * p.mean(i, inv));
            if (to >= 0) red[to * width + tx * V + i] = a;
        }
        __syncthreads();
        group_sums(red, lines, width, s.cg, s.slab_g, [&](int g, float v) { mu[g] = v * total; });
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float b = fold(s, seen ? p.square(i, k, inv, mu[(tx * V + i) / s.cg]) : 0.f);
            if (to >= 0) red[to * width + tx * V + i] = b;
        }
        __syncthreads();
        group_sums(red, lines, width, s.cg, s.slab_g, [&](int g, float v) { out(g, make_float2(mu[g], v)); });
    }
}

// ---- copies into a thread's own places of shared memory: they need no registers while they are under way, and no barrier ----------------------
template <class T, int V>
__device__ __forceinline__ void copy_in(uint32_t dst, const T *src) {
    if constexpr (V * sizeof(T) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else if constexpr (V * sizeof(T) == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
    else if constexpr (V * sizeof(T) == 4) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("st.shared.u16 [%0], %1;" ::"r"(dst), "h"(*(const uint16_t *)src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <class T, int V>
__device__ __forceinline__ NormVec<T, V> kept_vec(uint32_t addr) {
    NormVec<T, V> v;
    if constexpr (V * sizeof(T) == 16) {
        uint4 q;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(addr) : "memory");
        v.w = q;
    } else if constexpr (V * sizeof(T) == 8) {
        uint2 q;
        asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(q.x), "=r"(q.y) : "r"(addr) : "memory");
        v.w = q;
    } else if constexpr (V * sizeof(T) == 4) {
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v.w) : "r"(addr) : "memory");
    } else {
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v.w) : "r"(addr) : "memory");
    }
    return v;
}
// A column's pixels through a ring of kRing places, NT tensors side by side: f(its vectors) for pixel after pixel.  What is under way
// at a time, 48 KB a block, does not depend on how long a pixel takes; with a batch of loads in registers between one wait and the next the
// passes read 2.6 to 3.5 TB/s.
constexpr int kRing = 12, kBlocks1 = 3, kBlocks2 = 2;        // places; blocks of an SM, with one tensor and with two
template <class T, int V, int NT, bool COPIES = (V * sizeof(T) > 2)>
struct Ring {
    static constexpr int kPlaces = kRing / NT, kBatch = 2, kBatches = kPlaces / kBatch;
    static_assert(kBatches * kBatch == kPlaces, "whole batches");
    uint32_t slot;
    long long pitch;
    int mine;
    const T *from[NT];
    __device__ __forceinline__ void batch(int place, int left) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (i < left)
#pragma unroll
                for (int t = 0; t < NT; ++t) copy_in<T, V>(slot + ((place * kBatch + i) * NT + t) * (kThreads * 16), from[t]);
#pragma unroll
            for (int t = 0; t < NT; ++t) from[t] += pitch;
        }
        copies_commit();
    }
    __device__ __forceinline__ void start() {
#pragma unroll
        for (int b = 0; b < kBatches; ++b) batch(b, mine - b * kBatch);
    }
    template <class F>
    __device__ __forceinline__ void run(F &&f) {
        for (int left = mine; left > 0; left -= kPlaces) {
#pragma unroll
            for (int b = 0; b < kBatches; ++b) {
                copies_wait<kBatches - 1>();
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (b * kBatch + i < left) {
                        NormVec<T, V> v[NT];
#pragma unroll
                        for (int t = 0; t < NT; ++t) v[t] = kept_vec<T, V>(slot + ((b * kBatch + i) * NT + t) * (kThreads * 16));
                        f(v);
                    }
                batch(b, left - kPlaces - b * kBatch);
            }
        }
        copies_wait<0>();
    }
};
// The same for accesses of two bytes, which no asynchronous copy has: batches of loads in registers.
template <class T, int V, int NT>
struct Ring<T, V, NT, false> {
    static constexpr int kBatch = 16 / NT;
    uint32_t slot;
    long long pitch;
    int mine;
    const T *from[NT];
    __device__ __forceinline__ void start() {}
    template <class F>
    __device__ __forceinline__ void run(F &&f) {
        for (int left = mine; left > 0; left -= kBatch) {
            NormVec<T, V> v[kBatch][NT];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t) v[i][t].load(from[t] + (i < left ? i : 0) * pitch);
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (i < left) f(v[i]);
#pragma unroll
            for (int t = 0; t < NT; ++t) from[t] += kBatch * pitch;
        }
    }
};
constexpr int kRingBytes = kRing * kThreads * 16;

// ---- two passes -----------------------------------------------------------------------------------------------------------------------
// Mean and sum of squared distances of a cluster's runs of pixels, per group: part[(n runs + run) groups + g], runs = splits / cluster.
template <class T, int V>
__global__ void __launch_bounds__(kThreads, kBlocks1) group_norm_stats_kernel(const GroupNormShape s, const T *__restrict__ x, float2 *__restrict__ part) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ float red[kThreads * V];
    __shared__ float mu[kNormMaxSlabGroups];
    __shared__ float2 own[kNormMaxSlabGroups];
    const uint32_t slot = ptx::smem_u32(smem_raw) + threadIdx.x * 16;
    pdl_wait();
    pdl_launch_dependents();
    const int slab = blockIdx.y, split = blockIdx.x;
    const int n = s.n0 + blockIdx.z;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    const long long first = (long long)split * s.rows, rows = max(0LL, min(s.rows, s.pixels - first));
    const T *base = x + ((long long)n * s.pixels + first) * s.c + (long long)slab * s.slab_c;
    const int seen = ty < s.ty && ty < rows ? (int)((rows - ty + s.ty - 1) / s.ty) : 0;
    Moments m;
    Spread<T, V> sp;
    sp.none();
    if (seen > 0)
        for (int col = tx; col < s.cols; col += s.tx) {
            Ring<T, V, 1> ring{slot, (long long)s.ty * s.c, seen, {base + (long long)ty * s.c + (long long)col * V}};
            ring.start();
            bool begun = false;
            ring.run([&](const NormVec<T, V> (&v)[1]) {
                if (!begun) sp.first(v[0]);
                begun = true;
                sp.add(v[0]);
            });
            if (s.one_group) m.join(sp, seen);
        }
    block_moments(s, red, mu, s.one_group, m, sp, seen, (float)max(rows, 1LL), [&](int g, float2 v) { own[g] = v; });
    if (s.cluster > 1) ptx::cluster_sync_all(); else __syncthreads();
    const int rank = s.cluster > 1 ? (int)ptx::cluster_rank() : 0, run = split / s.cluster;
    if (rank == 0) {
        const long long from = (long long)run * s.cluster * s.rows;
        const float all = (float)max(1LL, min(s.rows * s.cluster, s.pixels - from));
        float2 *to = part + (((long long)n * (s.splits / s.cluster) + run) * s.g + (long long)slab * s.slab_g);
        for (int g = threadIdx.x; g < s.slab_g; g += kThreads) {
            float2 v = own[g];
            if (s.cluster > 1)
                v = join_runs(&own[g], s.cluster, all, (float)s.cg, [&](int b) { return (float)max(0LL, min(s.rows, s.pixels - from - b * s.rows)); });
            to[g] = v;
        }
    }
    if (s.cluster > 1) ptx::cluster_sync_all();                     // no block ends while another may read from it
}

// z = act(gamma (x - mean) r + beta).  Each block joins its groups' runs first; the first run's block writes saved.  Runs are taken from the last
// one on: what the pass before has read last is the likeliest in L2.
template <class T, int V, int ACT>
__global__ void __launch_bounds__(kThreads, kBlocks1) group_norm_apply_kernel(const GroupNormShape s, const T *__restrict__ x, const float *__restrict__ gamma,
                                                                       const float *__restrict__ beta, const float2 *__restrict__ part,
                                                                       float *__restrict__ saved, T *__restrict__ z) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ float2 stat[kNormMaxSlabGroups];
    pdl_wait();
    pdl_launch_dependents();
    const int slab = gridDim.y - 1 - blockIdx.y, split = s.splits - 1 - blockIdx.x;
    const int n = s.n0 + gridDim.z - 1 - blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, runs = s.splits / s.cluster;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    const long long first = (long long)split * s.rows, rows = min(s.rows, s.pixels - first);
    const int mine = ty < s.ty && ty < rows ? (int)((rows - ty + s.ty - 1) / s.ty) : 0;
    // from the last pixel on, too; the first ones are on their way while the runs are joined
    const long long last = ((long long)n * s.pixels + first + ty) * s.c + (long long)slab * s.slab_c + (mine - 1) * (long long)s.ty * s.c;
    const long long pitch = (long long)s.ty * s.c;
    Ring<T, V, 1> ring{ptx::smem_u32(smem_raw) + threadIdx.x * 16, -pitch, mine, {x + last + (long long)tx * V}};
    ring.start();
    const long long run_rows = s.rows * s.cluster;
    for (int g = warp; g < s.slab_g; g += kThreads / 32) {
        const float2 *p = part + (long long)n * runs * s.g + (long long)slab * s.slab_g + g;
        const float all = (float)s.pixels;
        float m = 0.f, q = 0.f;
        auto weight = [&](int i) { return (float)max(0LL, min(run_rows, s.pixels - i * run_rows)); };
        for (int i = lane; i < runs; i += 32) m = fmaf(weight(i) / all, p[(long long)i * s.g].x, m);
        m = warp_sum(m);
        for (int i = lane; i < runs; i += 32) {
            const float2 v = p[(long long)i * s.g];
            const float d = v.x - m;
            q += fmaf(weight(i) * s.cg * d, d, v.y);
        }
        q = warp_sum(q);
        if (lane == 0) {
            const float r = 1.f / sqrtf(q / (all * s.cg) + s.eps);
            stat[g] = make_float2(m, r);
            if (split == 0) {
                const long long to = (long long)n * s.g + (long long)slab * s.slab_g + g;
                saved[to] = m;
                saved[(long long)s.n * s.g + to] = r;
            }
        }
    }
    __syncthreads();
    if (mine == 0) return;
    for (int col = tx; col < s.cols; col += s.tx) {
        NormChannels<V, false> k;
        set_channels(k, col * V, s.cg, gamma + slab * s.slab_c, beta + slab * s.slab_c, [&](int g) { return stat[g]; });
        T *dst = z + last + (long long)col * V;
        if (col != tx) {
            ring.from[0] = x + last + (long long)col * V;
            ring.start();
        }
        ring.run([&](const NormVec<T, V> (&v)[1]) {
            norm_forward<T, V, ACT, false>(v[0], k).store_last(dst);
            dst -= pitch;
        });
    }
}

// Sums of the backward pass over a run of pixels: per channel dy and dy xhat, chan[(n splits + split) c + channel]; per group those two
// times gamma, part[(n splits + split) g + group].
template <class T, int V, int ACT>
__global__ void __launch_bounds__(kThreads, kBlocks2) group_norm_bwd_sums_kernel(const GroupNormShape s, const T *__restrict__ dz, const T *__restrict__ x,
                                                                          const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                          const float *__restrict__ saved, float2 *__restrict__ chan,
                                                                          float2 *__restrict__ part) {
    constexpr int P = (V + 1) / 2;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ float red_a[kThreads * V], red_b[kThreads * V];
    const uint32_t slot = ptx::smem_u32(smem_raw) + threadIdx.x * 16;
    pdl_wait();
    pdl_launch_dependents();
    const int slab = blockIdx.y, split = blockIdx.x;
    const int n = s.n0 + blockIdx.z;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx, line = table_row(s), lines = table_rows(s);
    const long long first = (long long)split * s.rows, rows = min(s.rows, s.pixels - first);
    const int mine = ty < s.ty && ty < rows ? (int)((rows - ty + s.ty - 1) / s.ty) : 0;
    const long long base = ((long long)n * s.pixels + first + ty) * s.c + (long long)slab * s.slab_c, pitch = (long long)s.ty * s.c;
    const float *mean_p = saved + (long long)n * s.g + (long long)slab * s.slab_g, *rstd_p = mean_p + (long long)s.n * s.g;
    const float *gamma_p = gamma + slab * s.slab_c, *beta_p = beta + slab * s.slab_c;
    const long long run = (long long)n * s.splits + split;
    const int width = s.tx * V;
    float ga = 0.f, gb = 0.f;                      // the only group's sums, where there is one (warp 0)
    for (int col0 = 0; col0 < s.cols; col0 += s.tx) {
        const int col = col0 + tx, cols = min(s.tx, s.cols - col0);
        f32x2 a[P], b[P];
#pragma unroll
        for (int i = 0; i < P; ++i) a[i] = b[i] = 0ull;
        if (mine > 0 && tx < cols) {
            NormChannels<V, false> k;
            set_channels(k, col * V, s.cg, gamma_p, beta_p, [&](int g) { return make_float2(__ldg(mean_p + g), __ldg(rstd_p + g)); });
            const NormExact exact{mean_p, rstd_p, gamma_p, beta_p, col * V, s.cg, near_zero(k)};
            Ring<T, V, 2> ring{slot, pitch, mine, {x + base + (long long)col * V, dz + base + (long long)col * V}};
            ring.start();
            ring.run([&](const NormVec<T, V> (&v)[2]) {
                f32x2 xc[P], dy[P];
                norm_grad<T, V, ACT, false>(v[0], v[1], k, exact, xc, dy);
#pragma unroll
                for (int i = 0; i < P; ++i) { a[i] = add2(a[i], dy[i]); b[i] = fma2(dy[i], xc[i], b[i]); }
            });
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float fa = fold(s, at<V>(a, i)), fb = fold(s, at<V>(b, i));
            if (line >= 0) { red_a[line * width + tx * V + i] = fa; red_b[line * width + tx * V + i] = fb; }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < cols * V; c += kThreads) {
            float sa = 0.f, sb = 0.f;
            for (int k = 0; k < lines; ++k) { sa += red_a[k * width + c]; sb += red_b[k * width + c]; }
            const int channel = col0 * V + c;
            sb *= __ldg(rstd_p + channel / s.cg);
            chan[run * s.c + slab * s.slab_c + channel] = make_float2(sa, sb);
            const float g = __ldg(gamma_p + channel);
            red_a[c] = g * sa;                       // (row 0 of this column has been read by this thread)
            red_b[c] = g * sb;
        }
        __syncthreads();
        const int size = s.slab_g == 1 ? cols * V : s.cg;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        for (int g = warp; g < s.slab_g; g += kThreads / 32) {
            float sa = 0.f, sb = 0.f;
            for (int i = lane; i < size; i += 32) { sa += red_a[g * size + i]; sb += red_b[g * size + i]; }
            sa = warp_sum(sa);
            sb = warp_sum(sb);
            if (s.slab_g == 1) { ga += sa; gb += sb; sa = ga; sb = gb; }
            if (lane == 0 && col0 + s.tx >= s.cols) part[run * s.g + (long long)slab * s.slab_g + g] = make_float2(sa, sb);
        }
        if (col0 + s.tx < s.cols) __syncthreads();
    }
}

// dgamma and dbeta: chan [runs][c] added up, 32 channels a block, in 64 bits: a batch has up to 2^30 runs, and after 2^24 like ones an fp32 sum
// stands still.  (Sixteen of a warp's in fp32 first, their loads under way together.)
__global__ void __launch_bounds__(1024) group_norm_finish_kernel(long long runs, int c, const float2 *__restrict__ chan, float *__restrict__ dgamma,
                                                                 float *__restrict__ dbeta) {
    __shared__ double2 sums[1024];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, channel = blockIdx.x * 32 + lane;
    double2 t = make_double2(0., 0.);
    if (channel < c) {
        constexpr int kBatch = 16;
        const float2 *p = chan + (long long)warp * c + channel;
        const long long pitch = 32LL * c;
        long long left = (runs - warp + 31) / 32;                // of this warp
        for (; left >= kBatch; left -= kBatch) {
            float2 v[kBatch];
#pragma unroll
            for (int q = 0; q < kBatch; ++q) { v[q] = *p; p += pitch; }
#pragma unroll
            for (int q = 1; q < kBatch; ++q) { v[0].x += v[q].x; v[0].y += v[q].y; }
            t.x += v[0].x;
            t.y += v[0].y;
        }
        float2 u = make_float2(0.f, 0.f);
#pragma unroll 4
        for (; left > 0; --left) {
            u.x += p->x;
            u.y += p->y;
            p += pitch;
        }
        t.x += u.x;
        t.y += u.y;
    }
    sums[threadIdx.x] = t;
    __syncthreads();
    if (warp == 0 && channel < c) {
        double2 v[4] = {t, sums[32 + lane], sums[64 + lane], sums[96 + lane]};
#pragma unroll
        for (int k = 4; k < 32; ++k) { v[k % 4].x += sums[k * 32 + lane].x; v[k % 4].y += sums[k * 32 + lane].y; }
        t.x = (v[0].x + v[1].x) + (v[2].x + v[3].x);
        t.y = (v[0].y + v[1].y) + (v[2].y + v[3].y);
        dbeta[channel] = (float)t.x;
        dgamma[channel] = (float)t.y;
    }
}

// dx = r (gamma dy - E[gamma dy] - xhat E[gamma dy xhat]) = scale dy + k1 + k2 (x - mean)
template <class T, int V, int ACT>
__global__ void __launch_bounds__(kThreads, kBlocks2) group_norm_bwd_apply_kernel(const GroupNormShape s, const T *__restrict__ dz, const T *__restrict__ x,
                                                                           const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                           const float *__restrict__ saved, const float2 *__restrict__ part,
                                                                           T *__restrict__ dx) {
    constexpr int P = (V + 1) / 2;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ float2 stat[kNormMaxSlabGroups];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int slab = gridDim.y - 1 - blockIdx.y, split = s.splits - 1 - blockIdx.x;
    const int n = s.n0 + gridDim.z - 1 - blockIdx.z;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    const long long first = (long long)split * s.rows, rows = min(s.rows, s.pixels - first), pitch = (long long)s.ty * s.c;
    const int mine = ty < s.ty && ty < rows ? (int)((rows - ty + s.ty - 1) / s.ty) : 0;
    const long long last = ((long long)n * s.pixels + first + ty) * s.c + (long long)slab * s.slab_c + (mine - 1) * pitch;
    Ring<T, V, 2> ring{ptx::smem_u32(smem_raw) + threadIdx.x * 16, -pitch, mine, {x + last + (long long)tx * V, dz + last + (long long)tx * V}};
    ring.start();
    const float *mean_p = saved + (long long)n * s.g + (long long)slab * s.slab_g, *rstd_p = mean_p + (long long)s.n * s.g;
    for (int g = warp; g < s.slab_g; g += kThreads / 32) {
        const float2 *p = part + (long long)n * s.splits * s.g + (long long)slab * s.slab_g + g;
        float sa = 0.f, sb = 0.f;
        for (int i = lane; i < s.splits; i += 32) { const float2 v = p[(long long)i * s.g]; sa += v.x; sb += v.y; }
        sa = warp_sum(sa);
        sb = warp_sum(sb);
        const float inv = 1.f / ((float)s.pixels * (float)s.cg), r = __ldg(rstd_p + g);
        if (lane == 0) stat[g] = make_float2(-sa * inv * r, -sb * inv * r * r);
    }
    __syncthreads();
    if (mine == 0) return;
    const float *gamma_p = gamma + slab * s.slab_c, *beta_p = beta + slab * s.slab_c;
    for (int col = tx; col < s.cols; col += s.tx) {
        NormChannels<V, false> k;
        set_channels(k, col * V, s.cg, gamma_p, beta_p, [&](int g) { return make_float2(__ldg(mean_p + g), __ldg(rstd_p + g)); });
        const NormExact exact{mean_p, rstd_p, gamma_p, beta_p, col * V, s.cg, near_zero(k)};
        f32x2 k1[P], k2[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const float2 u = stat[(col * V + 2 * i) / s.cg], w = V > 1 ? stat[(col * V + 2 * i + 1) / s.cg] : make_float2(0.f, 0.f);
            k1[i] = pair(u.x, w.x);
            k2[i] = pair(u.y, w.y);
        }
        const long long from = last + (long long)col * V;
        if (col != tx) {
            ring.from[0] = x + from;
            ring.from[1] = dz + from;
            ring.start();
        }
        T *to = dx + from;
        ring.run([&](const NormVec<T, V> (&in)[2]) {
            f32x2 xc[P], dy[P];
            norm_grad<T, V, ACT, false>(in[0], in[1], k, exact, xc, dy);
            NormVec<T, V> v;
#pragma unroll
            for (int i = 0; i < P; ++i) v.put(i, fma2(dy[i], k.scale[i], fma2(xc[i], k2[i], k1[i])));
            v.store_last(to);
            to -= pitch;
        });
    }
}

// ---- on chip --------------------------------------------------------------------------------------------------------------------------
// A block has the slab of a sample, or a run of its pixels and its cluster the slab; a thread keeps `keep` of them, 16 bytes each, in places
// of shared memory that are its own: the copies need no registers while they are under way and no barrier.  Blocks are as small as hold
// their pixels: many run on an SM, and one's copies are under way beside another's sums.
// ONE: all channels of a thread belong to one group.
template <class T, int ACT, bool ONE>
__global__ void __launch_bounds__(kMaxKeptThreads) group_norm_kept_fwd_kernel(const GroupNormShape s, const T *__restrict__ x,
                                                                              const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                              float *__restrict__ saved, T *__restrict__ z) {
    constexpr int V = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ float mu[kNormMaxSlabGroups];
    __shared__ float2 own[kNormMaxSlabGroups], stat[kNormMaxSlabGroups];
    const uint32_t step = blockDim.x * 16, kept = ptx::smem_u32(smem_raw) + threadIdx.x * 16;
    float *red = (float *)(smem_raw + (size_t)s.keep * step);
    const int split = blockIdx.x, slab = blockIdx.y;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    const int first = split * (int)s.rows, rows = max(0, min((int)s.rows, (int)s.pixels - first));
    const int mine = ty < s.ty && ty < rows ? (rows - ty + s.ty - 1) / s.ty : 0;
    const long long pitch = (long long)s.ty * s.c, inside = (long long)(first + ty) * s.c + (long long)slab * s.slab_c + tx * V;
    const float *gamma_p = gamma + slab * s.slab_c, *beta_p = beta + slab * s.slab_c;
    pdl_wait();
    pdl_launch_dependents();
    for (int n = blockIdx.z; n < s.n; n += gridDim.z) {                  // (more samples than a grid has)
        const T *from = x + n * s.pixels * s.c + inside;
        for (int k = 0; k < mine; ++k) copy_in<T, V>(kept + k * step, from + k * pitch);
        copies_commit();
        copies_wait<0>();
        Spread<T, V> sp;
        sp.none();
        if (mine > 0) sp.first(kept_vec<T, V>(kept));
#pragma unroll 4
        for (int k = 1; k < mine; ++k) sp.add(kept_vec<T, V>(kept + k * step));
        Moments m;
        if (ONE && mine > 0) m.join(sp, mine);
        block_moments(s, red, mu, ONE, m, sp, mine, (float)max(rows, 1), [&](int g, float2 v) { own[g] = v; });
        if (s.cluster > 1) ptx::cluster_sync_all(); else __syncthreads();
        for (int g = threadIdx.x; g < s.slab_g; g += blockDim.x) {
            float2 v = own[g];
            if (s.cluster > 1)
                v = join_runs(&own[g], s.cluster, (float)s.pixels, (float)s.cg,
                              [&](int b) { return (float)max(0, min((int)s.rows, (int)s.pixels - b * (int)s.rows)); });
            const float r = 1.f / sqrtf(v.y / ((float)s.pixels * (float)s.cg) + s.eps);
            stat[g] = make_float2(v.x, r);
            if (split == 0) {
                const long long to = (long long)n * s.g + (long long)slab * s.slab_g + g;
                saved[to] = v.x;
                saved[(long long)s.n * s.g + to] = r;
            }
        }
        __syncthreads();
        if (mine > 0) {
            NormChannels<V, ONE> ch;
            set_channels(ch, tx * V, s.cg, gamma_p, beta_p, [&](int g) { return stat[g]; });
            T *to = z + n * s.pixels * s.c + inside;
#pragma unroll 2
            for (int k = 0; k < mine; ++k) norm_forward<T, V, ACT, ONE>(kept_vec<T, V>(kept + k * step), ch).store(to + k * pitch);
        }
        if (s.cluster > 1) ptx::cluster_sync_all();               // no block ends, or sums the next sample, while another may read from it
    }
}

template <class T, int ACT, bool ONE>
__global__ void __launch_bounds__(kMaxKeptThreads) group_norm_kept_bwd_kernel(const GroupNormShape s, const T *__restrict__ dz, const T *__restrict__ x,
                                                                              const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                              const float *__restrict__ saved, float2 *__restrict__ chan,
                                                                              T *__restrict__ dx) {
    constexpr int V = 16 / (int)sizeof(T), P = V / 2;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ float2 own[kNormMaxSlabGroups], stat[kNormMaxSlabGroups];
    const uint32_t step = blockDim.x * 16, kept = ptx::smem_u32(smem_raw) + threadIdx.x * 16;      // x and dz of a pixel in turn
    const int split = blockIdx.x, slab = blockIdx.y, width = s.tx * V;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx, line = table_row(s), lines = table_rows(s);
    float *red_a = (float *)(smem_raw + (size_t)s.keep * 2 * step), *red_b = red_a + lines * width;
    const int first = split * (int)s.rows, rows = max(0, min((int)s.rows, (int)s.pixels - first));
    const int mine = ty < s.ty && ty < rows ? (rows - ty + s.ty - 1) / s.ty : 0;
    const long long pitch = (long long)s.ty * s.c, inside = (long long)(first + ty) * s.c + (long long)slab * s.slab_c + tx * V;
    const float *gamma_p = gamma + slab * s.slab_c, *beta_p = beta + slab * s.slab_c;
    pdl_wait();
    pdl_launch_dependents();
    for (int n = blockIdx.z; n < s.n; n += gridDim.z) {
        const long long sample = n * s.pixels * s.c + inside;
        for (int k = 0; k < mine; ++k) {
            copy_in<T, V>(kept + 2 * k * step, x + sample + k * pitch);
            copy_in<T, V>(kept + (2 * k + 1) * step, dz + sample + k * pitch);
        }
        copies_commit();
        const float *mean_p = saved + (long long)n * s.g + (long long)slab * s.slab_g, *rstd_p = mean_p + (long long)s.n * s.g;
        NormChannels<V, ONE> ch;
        f32x2 a[P], b[P];
        NormExact exact{mean_p, rstd_p, gamma_p, beta_p, tx * V, s.cg, 0.f};
        if (mine > 0) {
            set_channels(ch, tx * V, s.cg, gamma_p, beta_p, [&](int g) { return make_float2(__ldg(mean_p + g), __ldg(rstd_p + g)); });
            exact.near = near_zero(ch);
        }
#pragma unroll
        for (int i = 0; i < P; ++i) a[i] = b[i] = 0ull;
        copies_wait<0>();
#pragma unroll 2
        for (int k = 0; k < mine; ++k) {
            f32x2 xc[P], dy[P];
            norm_grad<T, V, ACT, ONE>(kept_vec<T, V>(kept + 2 * k * step), kept_vec<T, V>(kept + (2 * k + 1) * step), ch, exact, xc, dy);
#pragma unroll
            for (int i = 0; i < P; ++i) { a[i] = add2(a[i], dy[i]); b[i] = fma2(dy[i], xc[i], b[i]); }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float fa = fold(s, at<V>(a, i)), fb = fold(s, at<V>(b, i));
            if (line >= 0) { red_a[line * width + tx * V + i] = fa; red_b[line * width + tx * V + i] = fb; }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < width; c += blockDim.x) {
            float sa = 0.f, sb = 0.f;
            for (int k = 0; k < lines; ++k) { sa += red_a[k * width + c]; sb += red_b[k * width + c]; }
            sb *= __ldg(rstd_p + c / s.cg);
            chan[((long long)n * s.splits + split) * s.c + slab * s.slab_c + c] = make_float2(sa, sb);
            const float g = __ldg(gamma_p + c);
            red_a[c] = g * sa;                       // (row 0 of this column has been read by this thread)
            red_b[c] = g * sb;
        }
        __syncthreads();
        group_sums(red_a, 1, width, s.cg, s.slab_g, [&](int g, float v) { own[g].x = v; });
        group_sums(red_b, 1, width, s.cg, s.slab_g, [&](int g, float v) { own[g].y = v; });
        if (s.cluster > 1) ptx::cluster_sync_all(); else __syncthreads();
        for (int g = threadIdx.x; g < s.slab_g; g += blockDim.x) {
            float2 all = own[g];
            if (s.cluster > 1) {
                float2 v[kMaxCluster];
                cluster_pairs(&own[g], s.cluster, v);
                all = v[0];
#pragma unroll
                for (int k = 1; k < kMaxCluster; ++k)
                    if (k < s.cluster) { all.x += v[k].x; all.y += v[k].y; }
            }
            const float inv = 1.f / ((float)s.pixels * (float)s.cg), r = __ldg(rstd_p + g);
            stat[g] = make_float2(-all.x * inv * r, -all.y * inv * r * r);
        }
        __syncthreads();
        if (mine > 0) {
            f32x2 k1[ONE ? 1 : P], k2[ONE ? 1 : P];
#pragma unroll
            for (int i = 0; i < (ONE ? 1 : P); ++i) {
                const float2 f = stat[(tx * V + 2 * i) / s.cg], w = ONE ? f : stat[(tx * V + 2 * i + 1) / s.cg];
                k1[i] = pair(f.x, w.x);
                k2[i] = pair(f.y, w.y);
            }
#pragma unroll 2
            for (int k = 0; k < mine; ++k) {
                f32x2 xc[P], dy[P];
                norm_grad<T, V, ACT, ONE>(kept_vec<T, V>(kept + 2 * k * step), kept_vec<T, V>(kept + (2 * k + 1) * step), ch, exact, xc, dy);
                NormVec<T, V> v;
#pragma unroll
                for (int i = 0; i < P; ++i) v.put(i, fma2(dy[i], ch.scale[i], fma2(xc[i], k2[ONE ? 0 : i], k1[ONE ? 0 : i])));
                v.store(dx + sample + k * pitch);
            }
        }
        if (s.cluster > 1) ptx::cluster_sync_all();
    }
}

// Dynamic shared memory of a block: its pixels and its table of sums.
int kept_smem(const GroupNormShape &s, bool backward) {
    const int lines = s.fold ? s.threads / 32 : s.ty, wide = backward ? 2 * s.vec : s.one_group ? 1 : s.vec;
    return s.keep * s.threads * (backward ? 32 : 16) + lines * s.tx * wide * 4;
}
template <class K, class... Args>
cudaError_t launch_clusters(K kernel, const GroupNormShape &s, dim3 grid, int smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)s.threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = s.cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = s.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, s, args...);
}

// f(a value of the storage type, elements per access, activation)
template <class F>
cudaError_t dispatch(const GroupNormShape &s, F &&f) {
    using std::integral_constant;
    auto by_act = [&](auto t, auto v) {
        switch (s.act) {
            case CONVBN_ACT_RELU: return f(t, v, integral_constant<int, CONVBN_ACT_RELU>());
            case CONVBN_ACT_SILU: return f(t, v, integral_constant<int, CONVBN_ACT_SILU>());
            default: return f(t, v, integral_constant<int, CONVBN_ACT_NONE>());
        }
    };
    auto by_width = [&](auto t) {
        switch (s.vec * (int)sizeof(t)) {
            case 16: return by_act(t, integral_constant<int, 16 / (int)sizeof(t)>());
            case 8: return by_act(t, integral_constant<int, 8 / (int)sizeof(t)>());
            case 4: return by_act(t, integral_constant<int, 4 / (int)sizeof(t)>());
            default: return by_act(t, integral_constant<int, 1>());
        }
    };
    return s.dtype == CONVBN_F32 ? by_width(float()) : s.dtype == CONVBN_F16 ? by_width(__half()) : by_width(__nv_bfloat16());
}

// The narrowest slab of whole groups that starts on an access of s.vec elements and has 128 bytes a pixel, or as many as a block can take.
int slab_groups(const GroupNormShape &s, int es, int threads) {
    int groups = 0;
    for (int k = 1; k <= s.g && k <= kNormMaxSlabGroups; ++k) {
        if (s.g % k || k * s.cg % s.vec || (k > 1 && k * s.cg / s.vec > threads)) continue;
        groups = k;
        if ((long long)k * s.cg * es >= 128) break;
    }
    return groups;
}
void set_slab(GroupNormShape &s, int groups, int threads) {
    s.slab_g = groups;
    s.slab_c = groups * s.cg;
    s.cols = s.slab_c / s.vec;
    s.threads = threads;
    s.tx = s.cols < threads ? s.cols : threads;
    s.ty = threads / s.tx;
    s.one_group = groups == 1 || s.cg % s.vec == 0;
    s.fold = s.tx <= 32 && 32 % s.tx == 0;
}

// On chip: the fewest threads that hold the slab.
bool kept_plan(GroupNormShape &s, int es, bool backward) {
    if (s.vec * es != 16) return false;
    const int sms = device_sm_count(), most = kKept / (backward ? 32 : 16);
    for (int threads = 32; threads <= kMaxKeptThreads; threads *= 2) {
        const int groups = slab_groups(s, es, threads);
        if (!groups) continue;
        set_slab(s, groups, threads);
        // (few slabs: a cluster each)
        const long long units = (long long)(s.g / s.slab_g) * s.n, room = units * 2 <= sms ? std::min(sms / units, (long long)kMaxCluster) : 1;
        if (s.cols > threads || s.pixels > room * s.ty * most) continue;
        const long long splits = std::max(1LL, std::min(room, s.pixels / s.ty));
        s.splits = s.cluster = (int)splits;
        s.rows = (s.pixels + splits - 1) / splits;
        s.keep = (int)((s.rows + s.ty - 1) / s.ty);
        s.batch = std::min(s.n, 65535);
        return true;
    }
    return false;
}

}  // namespace

GroupNormShape group_norm_shape(const convbn_group_norm_desc *d, bool backward) {
    GroupNormShape s;
    s.n = d->n; s.c = d->c; s.g = d->groups; s.cg = d->c / d->groups; s.act = d->act; s.dtype = d->dtype;
    s.pixels = (long long)d->h * d->w;
    s.eps = (float)d->eps;
    s.n0 = 0;
    const int es = d->dtype == CONVBN_F32 ? 4 : 2;
    for (s.vec = 16 / es; s.c % s.vec || !slab_groups(s, es, kThreads); s.vec /= 2) {}       // (one element: one group always is)
    if (kept_plan(s, es, backward)) return s;
    s.keep = 0;
    set_slab(s, slab_groups(s, es, kThreads), kThreads);
    s.batch = std::min(s.n, kNormMaxBatch);
    // Runs of pixels: as many as blocks run at a time, each thread at least sixteen pixels.
    const long long units = (long long)(s.g / s.slab_g) * s.batch, most = (s.pixels + 16 * s.ty - 1) / (16 * s.ty);
    const long long room = (long long)(backward ? kBlocks2 : kBlocks1) * device_sm_count();
    long long splits = std::min(std::max(1LL, room / units), std::min(most, 1024LL));
    s.cluster = 1;
    if (!backward && splits > 8) { s.cluster = 8; splits -= splits % 8; }
    s.splits = (int)splits;
    s.rows = (s.pixels + splits - 1) / splits;
    if (s.cluster == 1) s.splits = (int)((s.pixels + s.rows - 1) / s.rows);
    return s;
}

// Two passes: [runs][groups] pairs.  Backward: [runs][channels] pairs behind them.
static long long runs_of(const GroupNormShape &s) { return (long long)s.n * s.splits; }
static size_t part_bytes(const GroupNormShape &s) { return s.keep ? 0 : align_up((size_t)runs_of(s) * s.g * sizeof(float2), 256); }
size_t group_norm_workspace(const GroupNormShape &s, bool backward) {
    const size_t bytes = part_bytes(s) + (backward ? align_up((size_t)runs_of(s) * s.c * sizeof(float2), 256) : 0);
    return bytes ? bytes : 256;
}

// f(share of the batch) for every launch's
template <class F>
static cudaError_t by_batch(const GroupNormShape &shape, F &&f) {
    GroupNormShape s = shape;
    cudaError_t e = cudaSuccess;
    for (int n0 = 0; n0 < shape.n && e == cudaSuccess; n0 += shape.batch) {
        s.n0 = n0;
        s.batch = shape.n - n0 < shape.batch ? shape.n - n0 : shape.batch;
        e = f(s);
    }
    return e;
}

cudaError_t launch_group_norm_fwd(const GroupNormShape &shape, const void *x, const float *gamma, const float *beta, void *z, float *saved,
                                  void *workspace, cudaStream_t st) {
    return dispatch(shape, [&](auto t, auto v, auto act) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, ACT = decltype(act)::value;
        const unsigned slabs = (unsigned)(shape.g / shape.slab_g);
        if constexpr (V * sizeof(T) == 16) {
            static PerDevice attr[2];
            if (shape.keep) {
                auto kernel = shape.one_group ? group_norm_kept_fwd_kernel<T, ACT, true> : group_norm_kept_fwd_kernel<T, ACT, false>;
                if (cudaError_t e = max_dynamic_smem_once(kernel, 200 * 1024, &attr[shape.one_group]); e != cudaSuccess) return e;
                return launch_clusters(kernel, shape, dim3((unsigned)shape.splits, slabs, (unsigned)shape.batch), kept_smem(shape, false), st,
                                       (const T *)x, gamma, beta, saved, (T *)z);
            }
        }
        return by_batch(shape, [&](const GroupNormShape &s) {
            const dim3 grid((unsigned)s.splits, slabs, (unsigned)s.batch);
            static PerDevice ring[2];
            cudaError_t e = max_dynamic_smem_once(group_norm_stats_kernel<T, V>, kRingBytes, &ring[0]);
            if (e == cudaSuccess) e = max_dynamic_smem_once(group_norm_apply_kernel<T, V, ACT>, kRingBytes, &ring[1]);
            if (e != cudaSuccess) return e;
            e = launch_clusters(group_norm_stats_kernel<T, V>, s, grid, kRingBytes, st, (const T *)x, (float2 *)workspace);
            if (e != cudaSuccess) return e;
            return launch_pdl(group_norm_apply_kernel<T, V, ACT>, grid, dim3(kThreads), kRingBytes, st, s, (const T *)x, gamma, beta, (const float2 *)workspace,
                              saved, (T *)z);
        });
    });
}

cudaError_t launch_group_norm_bwd(const GroupNormShape &shape, const void *dz, const void *x, const float *gamma, const float *beta,
                                  const float *saved, void *dx, float *dgamma, float *dbeta, void *workspace, cudaStream_t st) {
    float2 *part = (float2 *)workspace, *chan = (float2 *)((char *)workspace + part_bytes(shape));
    const cudaError_t e = dispatch(shape, [&](auto t, auto v, auto act) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, ACT = decltype(act)::value;
        const unsigned slabs = (unsigned)(shape.g / shape.slab_g);
        if constexpr (V * sizeof(T) == 16) {
            static PerDevice attr[2];
            if (shape.keep) {
                auto kernel = shape.one_group ? group_norm_kept_bwd_kernel<T, ACT, true> : group_norm_kept_bwd_kernel<T, ACT, false>;
                if (cudaError_t e = max_dynamic_smem_once(kernel, 200 * 1024, &attr[shape.one_group]); e != cudaSuccess) return e;
                return launch_clusters(kernel, shape, dim3((unsigned)shape.splits, slabs, (unsigned)shape.batch), kept_smem(shape, true), st,
                                       (const T *)dz, (const T *)x, gamma, beta, saved, chan, (T *)dx);
            }
        }
        return by_batch(shape, [&](const GroupNormShape &s) {
            const dim3 grid((unsigned)s.splits, slabs, (unsigned)s.batch);
            static PerDevice ring[2];
            cudaError_t e = max_dynamic_smem_once(group_norm_bwd_sums_kernel<T, V, ACT>, kRingBytes, &ring[0]);
            if (e == cudaSuccess) e = max_dynamic_smem_once(group_norm_bwd_apply_kernel<T, V, ACT>, kRingBytes, &ring[1]);
            if (e != cudaSuccess) return e;
            e = launch_pdl(group_norm_bwd_sums_kernel<T, V, ACT>, grid, dim3(kThreads), kRingBytes, st, s, (const T *)dz, (const T *)x, gamma, beta,
                                             saved, chan, part);
            if (e != cudaSuccess) return e;
            return launch_pdl(group_norm_bwd_apply_kernel<T, V, ACT>, grid, dim3(kThreads), kRingBytes, st, s, (const T *)dz, (const T *)x, gamma, beta, saved,
                              (const float2 *)part, (T *)dx);
        });
    });
    if (e != cudaSuccess) return e;
    return launch_pdl(group_norm_finish_kernel, dim3((unsigned)((shape.c + 31) / 32)), dim3(1024), 0, st, runs_of(shape), shape.c, (const float2 *)chan,
                      dgamma, dbeta);
}

}  // namespace convbn
