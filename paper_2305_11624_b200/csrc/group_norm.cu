// Group norm with its activation over channels-last activations, forward and backward (formulas: group_norm.cuh).
//
// Two passes each way.  The first sums, the second reads the same tensors again and writes.  A block takes a slab of channels (whole
// groups, 128 bytes of a pixel or more, so that every access of a warp is whole lines) of a run of pixels of one sample; a thread keeps its
// channels, so what belongs to a channel stays in registers.
#include "group_norm.cuh"
#include "sm100_ptx.cuh"

namespace convbn {

namespace {

constexpr int kThreads = 256;

// Sums of a block: of the elements that its warps hold in `red`, [rows][width] with `rows` thread rows; groups of `size` neighbours.
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <class F>
__device__ __forceinline__ void group_sums(const float *red, int rows, int width, int size, int groups, F &&out) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int g = warp; g < groups; g += kThreads / 32) {
        float s = 0.f;
        for (int i = lane; i < rows * size; i += 32) s += red[(i / size) * width + g * size + i % size];
        s = warp_sum(s);
        if (lane == 0) out(g, s);
    }
}

// Mean and sum of squared distances of a run of pixels, per group: part[(n splits + split) groups + g].
// Every thread sums distances from its channel's first value, which is one of the values: what those sums lose by rounding is small against
// the spread that the value itself brings in, however far the mean is from zero.
template <class T, int V>
__global__ void __launch_bounds__(kThreads) group_norm_stats_kernel(const GroupNormShape s, const T *__restrict__ x, float2 *__restrict__ part) {
    __shared__ float red[kThreads * V];
    __shared__ float mu[kNormMaxSlabGroups];
    pdl_wait();
    pdl_launch_dependents();
    const int slab = blockIdx.y, split = blockIdx.x;
    const int n = s.n0 + blockIdx.z;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    const long long first = (long long)split * s.rows, last = min(first + s.rows, s.pixels);
    const T *base = x + ((long long)n * s.pixels) * s.c + (long long)slab * s.slab_c;
    const bool live = ty < s.ty;
    float cnt = 0.f, mean = 0.f, m2 = 0.f;            // of all the thread's values (channels of one group)
    float ck[V], cs[V], cq[V];                        // per channel: first value, sums of distances and squares
    int seen = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) ck[i] = cs[i] = cq[i] = 0.f;
    for (int col = tx; col < s.cols; col += s.tx) {
        const T *p = base + (long long)col * V;
        seen = 0;
        long long r = first + ty;
        if (live && r < last) {
            NormVec<T, V> v;
            v.load(p + r * s.c);
            v.get(ck);
#pragma unroll
            for (int i = 0; i < V; ++i) cs[i] = cq[i] = 0.f;
            seen = 1;
            r += s.ty;
            constexpr int U = 4;
            for (; r + (long long)(U - 1) * s.ty < last; r += (long long)U * s.ty) {
                NormVec<T, V> u[U];
#pragma unroll
                for (int k = 0; k < U; ++k) u[k].load(p + (r + (long long)k * s.ty) * s.c);
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    float f[V];
                    u[k].get(f);
#pragma unroll
                    for (int i = 0; i < V; ++i) { const float d = f[i] - ck[i]; cs[i] += d; cq[i] = fmaf(d, d, cq[i]); }
                }
                seen += U;
            }
            for (; r < last; r += s.ty) {
                v.load(p + r * s.c);
                float f[V];
                v.get(f);
#pragma unroll
                for (int i = 0; i < V; ++i) { const float d = f[i] - ck[i]; cs[i] += d; cq[i] = fmaf(d, d, cq[i]); }
                ++seen;
            }
            if (s.one_group) {
                // the column's values, joined with what the thread has (Chan, Golub, LeVeque: pairwise updates of a variance)
                const float k = (float)seen, inv = 1.f / k;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) sum += fmaf(cs[i], inv, ck[i]);
                const float m = sum * (1.f / V);
                float q = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = fmaf(cs[i], inv, ck[i]) - m;
                    q += fmaf(-cs[i] * inv, cs[i], cq[i]) + k * d * d;
                }
                const float add = k * V, all = cnt + add, d = m - mean;
                mean += d * (add / all);
                m2 += q + d * d * (cnt * (add / all));
                cnt = all;
            }
        }
    }
    const long long rows = last - first;
    const float total = (float)rows * (float)s.cg;      // (an integer below 2^24 or rounded: the weights of a mean)
    float2 *out = part + (((long long)n * s.splits + split) * s.g + (long long)slab * s.slab_g);
    if (s.one_group) {
        // threads' columns of a group are neighbours: [ty][tx], V channels each
        const int per = s.slab_g == 1 ? s.tx : s.cg / V;
        if (live) red[ty * s.tx + tx] = cnt * mean;
        __syncthreads();
        group_sums(red, s.ty, s.tx, per, s.slab_g, [&](int g, float v) { mu[g] = v / total; });
        __syncthreads();
        const int g = s.slab_g == 1 ? 0 : tx / per;
        if (live) { const float d = mean - mu[g]; red[ty * s.tx + tx] = m2 + cnt * d * d; }
        __syncthreads();
        group_sums(red, s.ty, s.tx, per, s.slab_g, [&](int g, float v) { out[g] = make_float2(mu[g], v); });
    } else {
        const float k = (float)seen, inv = seen ? 1.f / k : 0.f;
        const int width = s.tx * V;
        if (live)
#pragma unroll
            for (int i = 0; i < V; ++i) red[ty * width + tx * V + i] = fmaf(k, ck[i], cs[i]);
        __syncthreads();
        group_sums(red, s.ty, width, s.cg, s.slab_g, [&](int g, float v) { mu[g] = v / total; });
        __syncthreads();
        if (live)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = fmaf(cs[i], inv, ck[i]) - mu[(tx * V + i) / s.cg];
                red[ty * width + tx * V + i] = fmaf(-cs[i] * inv, cs[i], cq[i]) + k * d * d;
            }
        __syncthreads();
        group_sums(red, s.ty, width, s.cg, s.slab_g, [&](int g, float v) { out[g] = make_float2(mu[g], v); });
    }
}

// z = act(gamma (x - mean) r + beta).  Each block joins its groups' runs first; the first run's block writes saved.
template <class T, int V, int ACT>
__global__ void __launch_bounds__(kThreads) group_norm_apply_kernel(const GroupNormShape s, const T *__restrict__ x, const float *__restrict__ gamma,
                                                                    const float *__restrict__ beta, const float2 *__restrict__ part,
                                                                    float *__restrict__ saved, T *__restrict__ z) {
    __shared__ float2 stat[kNormMaxSlabGroups];
    pdl_wait();
    pdl_launch_dependents();
    const int slab = blockIdx.y, split = blockIdx.x;
    const int n = s.n0 + blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int g = warp; g < s.slab_g; g += kThreads / 32) {
        const float2 *p = part + (long long)n * s.splits * s.g + (long long)slab * s.slab_g + g;
        const float all = (float)s.pixels;
        float m = 0.f;
        for (int i = lane; i < s.splits; i += 32) {
            const float rows = (float)min(s.rows, s.pixels - (long long)i * s.rows);
            m = fmaf(rows / all, p[(long long)i * s.g].x, m);
        }
        m = warp_sum(m);
        float q = 0.f;
        for (int i = lane; i < s.splits; i += 32) {
            const float rows = (float)min(s.rows, s.pixels - (long long)i * s.rows);
            const float2 v = p[(long long)i * s.g];
            const float d = v.x - m;
            q += fmaf(rows * s.cg * d, d, v.y);
        }
        q = warp_sum(q);
        if (lane == 0) {
            const float r = 1.f / sqrtf(q / (all * s.cg) + s.eps);
            stat[g] = make_float2(m, r);
            if (split == 0) {
                const long long at = (long long)n * s.g + (long long)slab * s.slab_g + g;
                saved[at] = m;
                saved[(long long)s.n * s.g + at] = r;
            }
        }
    }
    __syncthreads();
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    if (ty >= s.ty) return;
    const long long first = (long long)split * s.rows, last = min(first + s.rows, s.pixels);
    const long long base = ((long long)n * s.pixels) * s.c + (long long)slab * s.slab_c;
    for (int col = tx; col < s.cols; col += s.tx) {
        float sub[V], mul[V], add[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = col * V + i;
            const float2 st = stat[c / s.cg];
            sub[i] = st.x;
            mul[i] = __ldg(gamma + slab * s.slab_c + c) * st.y;
            add[i] = __ldg(beta + slab * s.slab_c + c);
        }
        const T *src = x + base + (long long)col * V;
        T *dst = z + base + (long long)col * V;
        auto one = [&](NormVec<T, V> v, long long r) {
            float f[V];
            v.get(f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = norm_act<ACT>(fmaf(f[i] - sub[i], mul[i], add[i]));
            v.put(f);
            v.store(dst + r * s.c);
        };
        constexpr int U = 4;
        long long r = first + ty;
        for (; r + (long long)(U - 1) * s.ty < last; r += (long long)U * s.ty) {
            NormVec<T, V> v[U];
#pragma unroll
            for (int k = 0; k < U; ++k) v[k].load_last(src + (r + (long long)k * s.ty) * s.c);
#pragma unroll
            for (int k = 0; k < U; ++k) one(v[k], r + (long long)k * s.ty);
        }
        for (; r < last; r += s.ty) {
            NormVec<T, V> v;
            v.load_last(src + r * s.c);
            one(v, r);
        }
    }
}

// Sums of the backward pass over a run of pixels: per channel dy and dy xhat, chan[(n splits + split) c + channel]; per group those two
// times gamma, part[(n splits + split) g + group].
template <class T, int V, int ACT>
__global__ void __launch_bounds__(kThreads) group_norm_bwd_sums_kernel(const GroupNormShape s, const T *__restrict__ dz, const T *__restrict__ x,
                                                                       const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                       const float *__restrict__ saved, float2 *__restrict__ chan,
                                                                       float2 *__restrict__ part) {
    __shared__ float red_a[kThreads * V], red_b[kThreads * V];
    pdl_wait();
    pdl_launch_dependents();
    const int slab = blockIdx.y, split = blockIdx.x;
    const int n = s.n0 + blockIdx.z;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    const bool live = ty < s.ty;
    const long long first = (long long)split * s.rows, last = min(first + s.rows, s.pixels);
    const long long base = ((long long)n * s.pixels) * s.c + (long long)slab * s.slab_c;
    const float *mean_p = saved + (long long)n * s.g + (long long)slab * s.slab_g, *rstd_p = mean_p + (long long)s.n * s.g;
    const long long run = (long long)n * s.splits + split;
    const int width = s.tx * V;
    float ga = 0.f, gb = 0.f;                      // the only group's sums, where there is one (thread 0)
    for (int col0 = 0; col0 < s.cols; col0 += s.tx) {
        const int col = col0 + tx, cols = min(s.tx, s.cols - col0);
        float a[V], b[V];
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = b[i] = 0.f;
        if (live && tx < cols) {
            float mean[V], rstd[V], gm[V], bt[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = col * V + i;
                mean[i] = __ldg(mean_p + c / s.cg);
                rstd[i] = __ldg(rstd_p + c / s.cg);
                gm[i] = __ldg(gamma + slab * s.slab_c + c);
                bt[i] = __ldg(beta + slab * s.slab_c + c);
            }
            const T *px = x + base + (long long)col * V, *pz = dz + base + (long long)col * V;
            auto one = [&](const NormVec<T, V> &vx, const NormVec<T, V> &vz) {
                float fx[V], fz[V];
                vx.get(fx);
                vz.get(fz);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xc = fx[i] - mean[i];
                    const float dy = norm_act_grad<ACT>(fz[i], xc, fx[i], mean[i], rstd[i], gm[i], gm[i] * rstd[i], bt[i]);
                    a[i] += dy;
                    b[i] = fmaf(dy, xc, b[i]);
                }
            };
            constexpr int U = 2;
            long long r = first + ty;
            for (; r + (long long)(U - 1) * s.ty < last; r += (long long)U * s.ty) {
                NormVec<T, V> vx[U], vz[U];
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    vx[k].load(px + (r + (long long)k * s.ty) * s.c);
                    vz[k].load(pz + (r + (long long)k * s.ty) * s.c);
                }
#pragma unroll
                for (int k = 0; k < U; ++k) one(vx[k], vz[k]);
            }
            for (; r < last; r += s.ty) {
                NormVec<T, V> vx, vz;
                vx.load(px + r * s.c);
                vz.load(pz + r * s.c);
                one(vx, vz);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) b[i] *= rstd[i];
        }
        if (live)
#pragma unroll
            for (int i = 0; i < V; ++i) { red_a[ty * width + tx * V + i] = a[i]; red_b[ty * width + tx * V + i] = b[i]; }
        __syncthreads();
        for (int c = threadIdx.x; c < cols * V; c += kThreads) {
            float sa = 0.f, sb = 0.f;
            for (int k = 0; k < s.ty; ++k) { sa += red_a[k * width + c]; sb += red_b[k * width + c]; }
            const int channel = slab * s.slab_c + col0 * V + c;
            chan[run * s.c + channel] = make_float2(sa, sb);
            const float g = __ldg(gamma + channel);
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

// dgamma and dbeta: chan [runs][c] added up, 32 channels a block.
__global__ void __launch_bounds__(1024) group_norm_finish_kernel(long long runs, int c, const float2 *__restrict__ chan, float *__restrict__ dgamma,
                                                                 float *__restrict__ dbeta) {
    __shared__ float2 sums[1024];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, channel = blockIdx.x * 32 + lane;
    float2 t = make_float2(0.f, 0.f);
    if (channel < c) {
#pragma unroll 4
        for (long long i = warp; i < runs; i += 32) {
            const float2 v = chan[i * c + channel];
            t.x += v.x;
            t.y += v.y;
        }
    }
    sums[threadIdx.x] = t;
    __syncthreads();
    if (warp == 0 && channel < c) {
        for (int k = 1; k < 32; ++k) { t.x += sums[k * 32 + lane].x; t.y += sums[k * 32 + lane].y; }
        dbeta[channel] = t.x;
        dgamma[channel] = t.y;
    }
}

// dx = r (gamma dy - E[gamma dy] - xhat E[gamma dy xhat]).
template <class T, int V, int ACT>
__global__ void __launch_bounds__(kThreads) group_norm_bwd_apply_kernel(const GroupNormShape s, const T *__restrict__ dz, const T *__restrict__ x,
                                                                        const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                        const float *__restrict__ saved, const float2 *__restrict__ part,
                                                                        T *__restrict__ dx) {
    __shared__ float2 stat[kNormMaxSlabGroups];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int slab = blockIdx.y, split = blockIdx.x;
    const int n = s.n0 + blockIdx.z;
    const float *mean_p = saved + (long long)n * s.g + (long long)slab * s.slab_g, *rstd_p = mean_p + (long long)s.n * s.g;
    for (int g = warp; g < s.slab_g; g += kThreads / 32) {
        const float2 *p = part + (long long)n * s.splits * s.g + (long long)slab * s.slab_g + g;
        float sa = 0.f, sb = 0.f;
        for (int i = lane; i < s.splits; i += 32) { const float2 v = p[(long long)i * s.g]; sa += v.x; sb += v.y; }
        sa = warp_sum(sa);
        sb = warp_sum(sb);
        const float inv = 1.f / ((float)s.pixels * (float)s.cg), r = __ldg(rstd_p + g);
        if (lane == 0) stat[g] = make_float2(sa * inv * r, sb * inv * r * r);
    }
    __syncthreads();
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    if (ty >= s.ty) return;
    const long long first = (long long)split * s.rows, last = min(first + s.rows, s.pixels);
    const long long base = ((long long)n * s.pixels) * s.c + (long long)slab * s.slab_c;
    for (int col = tx; col < s.cols; col += s.tx) {
        float mean[V], rstd[V], gm[V], bt[V], k1[V], k2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = col * V + i, g = c / s.cg;
            mean[i] = __ldg(mean_p + g);
            rstd[i] = __ldg(rstd_p + g);
            gm[i] = __ldg(gamma + slab * s.slab_c + c);
            bt[i] = __ldg(beta + slab * s.slab_c + c);
            k1[i] = stat[g].x;
            k2[i] = stat[g].y;
        }
        const long long at = base + (long long)col * V;
        auto one = [&](const NormVec<T, V> &vx, const NormVec<T, V> &vz, long long r) {
            float fx[V], fz[V];
            vx.get(fx);
            vz.get(fz);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xc = fx[i] - mean[i], scale = gm[i] * rstd[i];
                const float dy = norm_act_grad<ACT>(fz[i], xc, fx[i], mean[i], rstd[i], gm[i], scale, bt[i]);
                fx[i] = fmaf(dy, scale, fmaf(-xc, k2[i], -k1[i]));
            }
            NormVec<T, V> v;
            v.put(fx);
            v.store(dx + at + r * s.c);
        };
        constexpr int U = 2;
        long long r = first + ty;
        for (; r + (long long)(U - 1) * s.ty < last; r += (long long)U * s.ty) {
            NormVec<T, V> vx[U], vz[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                vx[k].load_last(x + at + (r + (long long)k * s.ty) * s.c);
                vz[k].load_last(dz + at + (r + (long long)k * s.ty) * s.c);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) one(vx[k], vz[k], r + (long long)k * s.ty);
        }
        for (; r < last; r += s.ty) {
            NormVec<T, V> vx, vz;
            vx.load_last(x + at + r * s.c);
            vz.load_last(dz + at + r * s.c);
            one(vx, vz, r);
        }
    }
}

// ---- one pass: a sample's slab is kept on chip by a cluster of blocks -----------------------------------------------------------------
// A block has a run of the sample's pixels, a thread `keep` of them, 16 bytes each, in places of shared memory that are its own: the copies
// need no registers while they are under way and no barrier.  Sums go over the cluster through shared memory.
constexpr int kFusedMax = 8;                   // blocks of a cluster
constexpr int kFusedBytes = 72 * 1024;         // of a block: three blocks an SM

__device__ __forceinline__ void copy16(void *dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ float2 ld_cluster_f2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

// ONE: all channels of a thread belong to one group.
template <class T, int ACT, bool ONE>
__global__ void __launch_bounds__(kThreads, 3) group_norm_fused_fwd_kernel(const GroupNormShape s, const T *__restrict__ x, const float *__restrict__ gamma,
                                                                           const float *__restrict__ beta, float *__restrict__ saved, T *__restrict__ z) {
    constexpr int V = 16 / (int)sizeof(T), W = ONE ? 1 : V;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    using Vec = NormVec<T, V>;
    Vec *kept = (Vec *)smem_raw + threadIdx.x;
    __shared__ float red[kThreads * W];
    __shared__ float mu[kNormMaxSlabGroups];
    __shared__ float2 part[kNormMaxSlabGroups], stat[kNormMaxSlabGroups];
    pdl_wait();
    pdl_launch_dependents();
    const int rank = blockIdx.x % s.splits, slab = blockIdx.x / s.splits, n = s.n0 + blockIdx.y;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    const int first = rank * (int)s.rows, rows = max(0, min((int)s.rows, (int)s.pixels - first));
    const long long base = ((long long)n * s.pixels + first) * s.c + (long long)slab * s.slab_c + tx * V;
    const int mine = ty < s.ty && ty < rows ? (rows - ty + s.ty - 1) / s.ty : 0;
    const long long pitch = (long long)s.ty * s.c;
    {
        const T *p = x + base + (long long)ty * s.c;
        for (int k = 0; k < mine; ++k, p += pitch) copy16(kept + k * kThreads, p);
    }
    const int group = ONE ? (s.slab_g == 1 ? 0 : tx * V / s.cg) : 0, per = ONE ? (s.slab_g == 1 ? s.tx : s.cg / V) : s.cg;
    const int width = s.tx * W;
    const float inv = rows > 0 ? 1.f / ((float)rows * (float)s.cg) : 0.f;
    copies_wait();
    // the block's means, then the distances from them
    float sum[W];
#pragma unroll
    for (int i = 0; i < W; ++i) sum[i] = 0.f;
#pragma unroll 4
    for (int k = 0; k < mine; ++k) {
        float f[V];
        kept[k * kThreads].get(f);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[ONE ? 0 : i] += f[i];
    }
    if (ty < s.ty)
#pragma unroll
        for (int i = 0; i < W; ++i) red[ty * width + tx * W + i] = sum[i];
    __syncthreads();
    group_sums(red, s.ty, width, per, s.slab_g, [&](int g, float v) { mu[g] = v * inv; });
    __syncthreads();
    float m[W];
#pragma unroll
    for (int i = 0; i < W; ++i) { m[i] = mu[ONE ? group : (tx * V + i) / s.cg]; sum[i] = 0.f; }
#pragma unroll 4
    for (int k = 0; k < mine; ++k) {
        float f[V];
        kept[k * kThreads].get(f);
#pragma unroll
        for (int i = 0; i < V; ++i) { const float d = f[i] - m[ONE ? 0 : i]; sum[ONE ? 0 : i] = fmaf(d, d, sum[ONE ? 0 : i]); }
    }
    if (ty < s.ty)
#pragma unroll
        for (int i = 0; i < W; ++i) red[ty * width + tx * W + i] = sum[i];
    __syncthreads();
    group_sums(red, s.ty, width, per, s.slab_g, [&](int g, float v) { part[g] = make_float2(mu[g], v); });
    if (s.splits > 1) ptx::cluster_sync_all(); else __syncthreads();
    for (int g = threadIdx.x; g < s.slab_g; g += kThreads) {
        // the blocks' runs joined (pairwise update of mean and squared distances)
        float2 all = part[g];
        if (s.splits > 1) {
            float cnt = 0.f;
            all = make_float2(0.f, 0.f);
            for (int b = 0; b < s.splits; ++b) {
                const float2 v = ld_cluster_f2(ptx::cluster_addr(&part[g], b));
                const float add = (float)max(0, min((int)s.rows, (int)s.pixels - b * (int)s.rows)), share = add / (cnt + add), d = v.x - all.x;
                all.x = fmaf(d, share, all.x);
                all.y += fmaf(d * d, cnt * share * (float)s.cg, v.y);
                cnt += add;
            }
        }
        const float r = 1.f / sqrtf(all.y / ((float)s.pixels * (float)s.cg) + s.eps);
        stat[g] = make_float2(all.x, r);
        if (rank == 0) {
            const long long at = (long long)n * s.g + (long long)slab * s.slab_g + g;
            saved[at] = all.x;
            saved[(long long)s.n * s.g + at] = r;
        }
    }
    if (s.splits > 1) ptx::cluster_arrive_started();             // (done with the others' shared memory)
    __syncthreads();
    if (mine > 0) {
        float sub[W], mul[V], add[V];
        const int c0 = slab * s.slab_c + tx * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float2 st = stat[ONE ? group : (tx * V + i) / s.cg];
            sub[ONE ? 0 : i] = st.x;
            mul[i] = __ldg(gamma + c0 + i) * st.y;
            add[i] = __ldg(beta + c0 + i);
        }
        T *p = z + base + (long long)ty * s.c;
#pragma unroll 2
        for (int k = 0; k < mine; ++k, p += pitch) {
            Vec v = kept[k * kThreads];
            float f[V];
            v.get(f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = norm_act<ACT>(fmaf(f[i] - sub[ONE ? 0 : i], mul[i], add[i]));
            v.put(f);
            v.store(p);
        }
    }
    if (s.splits > 1) ptx::cluster_wait_started();               // no block ends while another may read from it
}

template <class T, int ACT, bool ONE>
__global__ void __launch_bounds__(kThreads, 2) group_norm_fused_bwd_kernel(const GroupNormShape s, const T *__restrict__ dz, const T *__restrict__ x,
                                                                           const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                           const float *__restrict__ saved, float2 *__restrict__ chan,
                                                                           T *__restrict__ dx) {
    constexpr int V = 16 / (int)sizeof(T), W = ONE ? 1 : V;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    using Vec = NormVec<T, V>;
    Vec *kept = (Vec *)smem_raw + threadIdx.x;                   // x and dz of a pixel in turn
    __shared__ float red_a[kThreads * V], red_b[kThreads * V];
    __shared__ float2 part[kNormMaxSlabGroups], stat[kNormMaxSlabGroups];
    pdl_wait();
    pdl_launch_dependents();
    const int rank = blockIdx.x % s.splits, slab = blockIdx.x / s.splits, n = s.n0 + blockIdx.y;
    const int tx = threadIdx.x % s.tx, ty = threadIdx.x / s.tx;
    const int first = rank * (int)s.rows, rows = max(0, min((int)s.rows, (int)s.pixels - first));
    const long long base = ((long long)n * s.pixels + first) * s.c + (long long)slab * s.slab_c + tx * V;
    const int mine = ty < s.ty && ty < rows ? (rows - ty + s.ty - 1) / s.ty : 0;
    const long long pitch = (long long)s.ty * s.c;
    {
        long long at = base + (long long)ty * s.c;
        for (int k = 0; k < mine; ++k, at += pitch) {
            copy16(kept + 2 * k * kThreads, x + at);
            copy16(kept + (2 * k + 1) * kThreads, dz + at);
        }
    }
    float mean[W], rstd[W], gm[V], bt[V], a[V], b[V];
    const int c0 = slab * s.slab_c + tx * V;
    const float *mean_p = saved + (long long)n * s.g + (long long)slab * s.slab_g, *rstd_p = mean_p + (long long)s.n * s.g;
    if (ty < s.ty) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = (tx * V + i) / s.cg;
            if (!ONE || i == 0) { mean[ONE ? 0 : i] = __ldg(mean_p + g); rstd[ONE ? 0 : i] = __ldg(rstd_p + g); }
            gm[i] = __ldg(gamma + c0 + i);
            bt[i] = __ldg(beta + c0 + i);
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = b[i] = 0.f;
    copies_wait();
#pragma unroll 2
    for (int k = 0; k < mine; ++k) {
        float fx[V], fz[V];
        kept[2 * k * kThreads].get(fx);
        kept[(2 * k + 1) * kThreads].get(fz);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float mn = mean[ONE ? 0 : i], rs = rstd[ONE ? 0 : i], xc = fx[i] - mn;
            const float dy = norm_act_grad<ACT>(fz[i], xc, fx[i], mn, rs, gm[i], gm[i] * rs, bt[i]);
            a[i] += dy;
            b[i] = fmaf(dy, xc, b[i]);
        }
    }
    const int width = s.tx * V;
    if (ty < s.ty)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            red_a[ty * width + tx * V + i] = a[i];
            red_b[ty * width + tx * V + i] = mine > 0 ? b[i] * rstd[ONE ? 0 : i] : 0.f;
        }
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += kThreads) {
        float sa = 0.f, sb = 0.f;
        for (int k = 0; k < s.ty; ++k) { sa += red_a[k * width + c]; sb += red_b[k * width + c]; }
        chan[((long long)n * s.splits + rank) * s.c + slab * s.slab_c + c] = make_float2(sa, sb);
        const float g = __ldg(gamma + slab * s.slab_c + c);
        red_a[c] = g * sa;                       // (row 0 of this column has been read by this thread)
        red_b[c] = g * sb;
    }
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int g = warp; g < s.slab_g; g += kThreads / 32) {
        float sa = 0.f, sb = 0.f;
        for (int i = lane; i < s.cg; i += 32) { sa += red_a[g * s.cg + i]; sb += red_b[g * s.cg + i]; }
        sa = warp_sum(sa);
        sb = warp_sum(sb);
        if (lane == 0) part[g] = make_float2(sa, sb);
    }
    if (s.splits > 1) ptx::cluster_sync_all(); else __syncthreads();
    for (int g = threadIdx.x; g < s.slab_g; g += kThreads) {
        float2 all = part[g];
        if (s.splits > 1) {
            all = make_float2(0.f, 0.f);
            for (int k = 0; k < s.splits; ++k) {
                const float2 v = ld_cluster_f2(ptx::cluster_addr(&part[g], k));
                all.x += v.x;
                all.y += v.y;
            }
        }
        const float inv = 1.f / ((float)s.pixels * (float)s.cg), r = __ldg(rstd_p + g);
        stat[g] = make_float2(all.x * inv * r, all.y * inv * r * r);
    }
    if (s.splits > 1) ptx::cluster_arrive_started();
    __syncthreads();
    if (mine > 0) {
        float k1[W], k2[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float2 st = stat[(tx * V + i) / s.cg];
            k1[i] = st.x;
            k2[i] = st.y;
        }
        T *p = dx + base + (long long)ty * s.c;
#pragma unroll 2
        for (int k = 0; k < mine; ++k, p += pitch) {
            float fx[V], fz[V];
            kept[2 * k * kThreads].get(fx);
            kept[(2 * k + 1) * kThreads].get(fz);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int o = ONE ? 0 : i;
                const float xc = fx[i] - mean[o], scale = gm[i] * rstd[o];
                const float dy = norm_act_grad<ACT>(fz[i], xc, fx[i], mean[o], rstd[o], gm[i], scale, bt[i]);
                fx[i] = fmaf(dy, scale, fmaf(-xc, k2[o], -k1[o]));
            }
            Vec v;
            v.put(fx);
            v.store(p);
        }
    }
    if (s.splits > 1) ptx::cluster_wait_started();
}

template <class K, class... Args>
cudaError_t launch_fused(K kernel, PerDevice *attr, const GroupNormShape &s, int per_pixel, cudaStream_t st, Args... args) {
    const int smem = s.keep * kThreads * per_pixel;
    if (cudaError_t e = max_dynamic_smem_once(kernel, kFusedBytes, attr); e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(s.splits * (s.g / s.slab_g)), (unsigned)s.batch);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = s.splits;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = s.splits > 1 ? 2 : 1;
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

}  // namespace

GroupNormShape group_norm_shape(const convbn_group_norm_desc *d, bool backward) {
    GroupNormShape s;
    s.n = d->n; s.c = d->c; s.g = d->groups; s.cg = d->c / d->groups; s.act = d->act; s.dtype = d->dtype;
    s.pixels = (long long)d->h * d->w;
    s.eps = (float)d->eps;
    const int es = d->dtype == CONVBN_F32 ? 4 : 2;
    // The widest access that rows allow, and the narrowest slab of whole groups that starts on such an access and has 128 bytes a pixel, or
    // as many as a block can take.
    for (s.vec = 16 / es;; s.vec /= 2) {
        if (s.c % s.vec) continue;
        s.slab_g = 0;
        for (int k = 1; k <= s.g && k <= kNormMaxSlabGroups; ++k) {
            if (s.g % k || k * s.cg % s.vec || (k > 1 && k * s.cg / s.vec > kThreads)) continue;
            s.slab_g = k;
            if ((long long)k * s.cg * es >= 128) break;
        }
        if (s.slab_g) break;                       // (one element: k = 1 always is)
    }
    s.slab_c = s.slab_g * s.cg;
    s.cols = s.slab_c / s.vec;
    s.tx = s.cols < kThreads ? s.cols : kThreads;
    s.ty = kThreads / s.tx;
    s.one_group = s.slab_g == 1 || s.cg % s.vec == 0;
    s.n0 = 0;
    s.batch = s.n;
    // Kept on chip: as few blocks as hold the sample's slab, more of them where that leaves SMs idle.
    const long long slabs = s.g / s.slab_g;
    const int sms = device_sm_count(), per_pixel = backward ? 32 : 16, most_kept = kFusedBytes / (kThreads * per_pixel);
    s.keep = 0;
    if (s.vec * es == 16 && s.cols <= kThreads && s.pixels <= (long long)kFusedMax * most_kept * s.ty) {
        int splits = (int)((s.pixels + (long long)most_kept * s.ty - 1) / ((long long)most_kept * s.ty));
        while (splits < kFusedMax && slabs * s.n * splits < 4LL * sms && s.pixels > 2LL * s.ty * splits) ++splits;
        s.rows = (s.pixels + splits - 1) / splits;
        s.splits = (int)((s.pixels + s.rows - 1) / s.rows);
        s.keep = (int)((s.rows + s.ty - 1) / s.ty);
        return s;
    }
    // Runs of pixels: four blocks an SM over the whole batch, each thread at least eight pixels.
    const long long want = (4LL * sms + slabs * s.n - 1) / (slabs * s.n);
    const long long most = (s.pixels + 8 * s.ty - 1) / (8 * s.ty);
    s.splits = (int)(want < most ? want : most);
    if (s.splits > 1024) s.splits = 1024;
    s.rows = (s.pixels + s.splits - 1) / s.splits;
    s.splits = (int)((s.pixels + s.rows - 1) / s.rows);
    return s;
}

// Two passes: [runs][groups] pairs.  Backward: [runs][channels] pairs behind them.
size_t group_norm_workspace(const GroupNormShape &s, bool backward) {
    const size_t runs = (size_t)s.n * s.splits;
    return align_up(runs * s.g * sizeof(float2), 256) + (backward ? align_up(runs * s.c * sizeof(float2), 256) : 0);
}

// f(first sample, samples) for every launch's share of the batch
template <class F>
static cudaError_t by_batch(const GroupNormShape &shape, F &&f) {
    GroupNormShape s = shape;
    cudaError_t e = cudaSuccess;
    for (int n0 = 0; n0 < shape.n && e == cudaSuccess; n0 += kNormMaxBatch) {
        s.n0 = n0;
        s.batch = shape.n - n0 < kNormMaxBatch ? shape.n - n0 : kNormMaxBatch;
        e = f(s);
    }
    return e;
}

cudaError_t launch_group_norm_fwd(const GroupNormShape &shape, const void *x, const float *gamma, const float *beta, void *z, float *saved,
                                  void *workspace, cudaStream_t st) {
    return dispatch(shape, [&](auto t, auto v, auto act) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, ACT = decltype(act)::value;
        if constexpr (V * sizeof(T) == 16) {
            static PerDevice attr[2];
            if (shape.keep)
                return by_batch(shape, [&](const GroupNormShape &s) {
                    auto kernel = s.one_group ? group_norm_fused_fwd_kernel<T, ACT, true> : group_norm_fused_fwd_kernel<T, ACT, false>;
                    return launch_fused(kernel, &attr[s.one_group], s, 16, st, (const T *)x, gamma, beta, saved, (T *)z);
                });
        }
        return by_batch(shape, [&](const GroupNormShape &s) {
            const dim3 grid((unsigned)s.splits, (unsigned)(s.g / s.slab_g), (unsigned)s.batch);
            const cudaError_t e = launch_pdl(group_norm_stats_kernel<T, V>, grid, dim3(kThreads), 0, st, s, (const T *)x, (float2 *)workspace);
            if (e != cudaSuccess) return e;
            return launch_pdl(group_norm_apply_kernel<T, V, ACT>, grid, dim3(kThreads), 0, st, s, (const T *)x, gamma, beta, (const float2 *)workspace,
                              saved, (T *)z);
        });
    });
}

cudaError_t launch_group_norm_bwd(const GroupNormShape &shape, const void *dz, const void *x, const float *gamma, const float *beta,
                                  const float *saved, void *dx, float *dgamma, float *dbeta, void *workspace, cudaStream_t st) {
    float2 *part = (float2 *)workspace;
    float2 *chan = (float2 *)((char *)workspace + align_up((size_t)shape.n * shape.splits * shape.g * sizeof(float2), 256));
    const cudaError_t e = dispatch(shape, [&](auto t, auto v, auto act) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, ACT = decltype(act)::value;
        if constexpr (V * sizeof(T) == 16) {
            static PerDevice attr[2];
            if (shape.keep)
                return by_batch(shape, [&](const GroupNormShape &s) {
                    auto kernel = s.one_group ? group_norm_fused_bwd_kernel<T, ACT, true> : group_norm_fused_bwd_kernel<T, ACT, false>;
                    return launch_fused(kernel, &attr[s.one_group], s, 32, st, (const T *)dz, (const T *)x, gamma, beta, saved, chan, (T *)dx);
                });
        }
        return by_batch(shape, [&](const GroupNormShape &s) {
            const dim3 grid((unsigned)s.splits, (unsigned)(s.g / s.slab_g), (unsigned)s.batch);
            const cudaError_t e = launch_pdl(group_norm_bwd_sums_kernel<T, V, ACT>, grid, dim3(kThreads), 0, st, s, (const T *)dz, (const T *)x, gamma, beta,
                                             saved, chan, part);
            if (e != cudaSuccess) return e;
            return launch_pdl(group_norm_bwd_apply_kernel<T, V, ACT>, grid, dim3(kThreads), 0, st, s, (const T *)dz, (const T *)x, gamma, beta, saved,
                              (const float2 *)part, (T *)dx);
        });
    });
    if (e != cudaSuccess) return e;
    return launch_pdl(group_norm_finish_kernel, dim3((unsigned)((shape.c + 31) / 32)), dim3(1024), 0, st, (long long)shape.n * shape.splits, shape.c,
                      (const float2 *)chan, dgamma, dbeta);
}

}  // namespace convbn
