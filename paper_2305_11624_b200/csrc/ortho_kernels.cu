// Orthogonal updates (formulas, pairs of halves, tiles: ortho.cuh): the matrices' norms, their way into tiles, and the products.
#include <algorithm>

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
    // A, R, then, where X is long, B and Q in its two places
    __host__ __device__ long long a() const { return 4 * x_bytes; }
    __host__ __device__ long long r() const { return 4 * x_bytes + 2 * s_bytes; }
    __host__ __device__ long long b() const { return 4 * x_bytes + 4 * s_bytes; }
    __host__ __device__ long long q(int which) const { return 4 * x_bytes + (6 + 2 * which) * s_bytes; }
    __host__ __device__ long long parts(bool wide) const { return 4 * x_bytes + (wide ? 10 : 4) * s_bytes; }       // fp32 pieces of A's tiles, 64 KB each
};
// Elements that a block sums the squares of: few enough for a matrix to fill the SMs, and no more pieces than its tiles' blocks read again at ease.
__host__ __device__ inline int ortho_chunk_of(const OrthoItem &it) { return (long long)it.rows * it.cols <= 1 << 22 ? 4096 : 16384; }
__host__ __device__ inline int ortho_chunks(const OrthoItem &it) {
    const int chunk = ortho_chunk_of(it);
    return (int)(((long long)it.rows * it.cols + chunk - 1) / chunk);
}
__host__ __device__ inline int ortho_lower(int rt, int ct) { const int d = rt < ct ? rt : ct; return d * (d + 1) / 2; }
__host__ __device__ inline long long ortho_sums_at(const OrthoItem &it) {
    const long long parts = it.splits > 1 ? (long long)ortho_lower(it.rt, it.ct) * it.splits * 65536 : 0;
    return OrthoPlace(it.rt, it.ct).parts(it.wide) + parts;
}
// In front of the matrices: [tasks taken | warps' shares done, per matrix | tickets of A's pieces, eight per tile], ints.
__host__ __device__ inline int ortho_words(const OrthoTable &t) { return 1 + t.matrices + 8 * t.squares; }

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

// Four elements from `at` on as one access (vec), or one by one, those from `left` on zero.
template <class T>
__device__ __forceinline__ float4 read4(const T *p, bool vec, int left) {
    float f[4] = {0.f, 0.f, 0.f, 0.f};
    if (vec && left >= 4) {
        if constexpr (sizeof(T) == 4) return *(const float4 *)p;
        else {
            const uint2 q = *(const uint2 *)p;
            const T *t = (const T *)&q;
            return make_float4(to_f32(t[0]), to_f32(t[1]), to_f32(t[2]), to_f32(t[3]));
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) f[e] = to_f32(p[e]);
    return make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void write4(float *p, bool vec, int left, float4 v) {
    if (vec && left >= 4) { *(float4 *)p = v; return; }
    const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) p[e] = f[e];
}
// Whether groups of four elements from multiples of four on lie on their boundary.
__device__ __forceinline__ bool ortho_vec(const OrthoTable &tab, const OrthoItem &it, int elem, long long base) {
    const uint64_t g = (uint64_t)it.g, v = tab.muon ? (uint64_t)it.momentum : 0;
    return g % (4 * elem) == 0 && v % 16 == 0 && base % 4 == 0;
}
__device__ __forceinline__ float4 fma4(float a, float4 b, float4 c) {
    return make_float4(fmaf(a, b.x, c.x), fmaf(a, b.y, c.y), fmaf(a, b.z, c.z), fmaf(a, b.w, c.w));
}

// Sums of squares of a chunk of a matrix's elements, in 64 bits (a gradient's squares leave fp32's range); muon: the momentum's step on the way.
// (Four accesses of a thread on their way; one element at a time the ResNet-50's layers took 80 us.)
template <class T>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const __grid_constant__ OrthoTable tab, uint8_t *__restrict__ ws) {
    __shared__ double part[8];
    pdl_wait();
    pdl_launch_dependents();
    const int task = blockIdx.x;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < ortho_words(tab); i += gridDim.x * 256) ((int *)ws)[i] = 0;
    const OrthoItem &it = tab.item[find_item(tab, task, [](const OrthoItem &i) { return i.first_sum; })];
    const int chunks = ortho_chunks(it), chunk = ortho_chunk_of(it), local = task - it.first_sum, copy = local / chunks, at = local - copy * chunks;
    const long long size = (long long)it.rows * it.cols, from = (long long)at * chunk, base = copy * size + from;
    const int n = (int)min((long long)chunk, size - from);
    const bool vec = ortho_vec(tab, it, tab.muon ? 4 : sizeof(T), base);
    double s = 0.;
    auto square = [&](float4 u) { s += (double)u.x * u.x + (double)u.y * u.y + (double)u.z * u.z + (double)u.w * u.w; };
    for (int i0 = threadIdx.x * 4; i0 < n; i0 += 4096) {
        float4 g[4], v[4];
        if (tab.muon) {
            const float *gp = (const float *)it.g + base;
            float *vp = it.momentum + base;
#pragma unroll
            for (int k = 0; k < 4; ++k) { g[k] = read4(gp + i0 + k * 1024, vec, n - i0 - k * 1024); v[k] = read4(vp + i0 + k * 1024, vec, n - i0 - k * 1024); }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = fma4(tab.momentum, v[k], g[k]);
                write4(vp + i0 + k * 1024, vec, n - i0 - k * 1024, v[k]);
                square(tab.nesterov ? fma4(tab.momentum, v[k], g[k]) : v[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) g[k] = read4((const T *)it.g + base + i0 + k * 1024, vec, n - i0 - k * 1024);
#pragma unroll
            for (int k = 0; k < 4; ++k) square(g[k]);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) s += part[i];
        ((double *)(ws + it.base + copy * it.bytes + ortho_sums_at(it)))[at] = s;
    }
}

// A tile of X = G / (|G| + eps), zeros beyond the matrix.  A thread has four columns of eight rows, which are on their way while the sums are
// added up.
template <class T>
__global__ void __launch_bounds__(256) ortho_tile_kernel(const __grid_constant__ OrthoTable tab, uint8_t *__restrict__ ws) {
    __shared__ double part[8];
    __shared__ OrthoScaling scaling;
    pdl_wait();
    pdl_launch_dependents();
    const int task = blockIdx.x;
    const OrthoItem &it = tab.item[find_item(tab, task, [](const OrthoItem &i) { return i.first_tile; })];
    const int per = it.rt * it.ct * 2, local = task - it.first_tile, copy = local / per, tile = local - copy * per;
    const OrthoPlace place(it.rt, it.ct);
    uint8_t *m = ws + it.base + copy * it.bytes;
    const double *sums = (const double *)(m + ortho_sums_at(it));
    const int row0 = tile / (2 * it.ct) * 128 + (threadIdx.x >> 4), col0 = tile % (2 * it.ct) * 64 + (threadIdx.x & 15) * 4;
    const long long base = copy * ((long long)it.rows * it.cols);
    const bool vec = ortho_vec(tab, it, tab.muon ? 4 : sizeof(T), base) && it.cols % 4 == 0;
    float4 u[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int r = row0 + 16 * k, left = r < it.rows ? it.cols - col0 : 0;
        const long long from = base + (long long)(r < it.rows ? r : 0) * it.cols + (left > 0 ? col0 : 0);
        if (!tab.muon) u[k] = read4((const T *)it.g + from, vec, left);
        else if (!tab.nesterov) u[k] = read4((const float *)it.momentum + from, vec, left);
        else u[k] = fma4(tab.momentum, read4((const float *)it.momentum + from, vec, left), read4((const float *)it.g + from, vec, left));
    }
    double s = 0.;
    for (int i = threadIdx.x; i < ortho_chunks(it); i += 256) s += sums[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = part[0];
        for (int i = 1; i < 8; ++i) s += part[i];
        scaling = OrthoScaling::of(s, tab.eps);
    }
    __syncthreads();
    const OrthoScaling scaled = scaling;
    uint8_t *hi = m + place.x(0) + (long long)tile * kOrthoTile, *lo = hi + place.x_bytes;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float x[4] = {scaled(u[k].x), scaled(u[k].y), scaled(u[k].z), scaled(u[k].w)};
        __half2 h[2], l[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            h[e] = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
            const float2 back = __half22float2(h[e]);
            l[e] = __floats2half2_rn(x[2 * e] - back.x, x[2 * e + 1] - back.y);
        }
        const uint32_t at = ortho_chunk((threadIdx.x >> 4) + 16 * k, (threadIdx.x & 15) >> 1) + (threadIdx.x & 1) * 8;
        *(uint2 *)(hi + at) = *(const uint2 *)h;
        *(uint2 *)(lo + at) = *(const uint2 *)l;
    }
}

// ---- products ---------------------------------------------------------------------------------------------------------------------
// All products of all steps in one launch (what they are: ortho.cuh).  CTA = 10 warps: 0 takes tasks and loads, 1 MMA issuer and owner of tensor
// memory, 2-9 epilogue.
// A task is a 128 x 128 (or 128 x 64) tile of a result (or a piece of the k of one of A's); k in steps of 64.  A step's four tiles (hi and lo of
// both operands) are 64 KB and feed twelve MMAs of one shape: hi hi into one half of the accumulator's 256 columns, hi lo and lo hi into the other.
// MMAs keep the order of issue only where accumulator and shape are the same, so hi of A with hi and lo of B side by side, one MMA instead of
// two, would need columns that lo hi does not touch.  128 x 64 tiles have them, and gain (A's rows come once less from shared memory: 512 x 4608
// 194 us instead of 200); 128 x 128 ones do not, and would not: two 2048 x 8192 take 2126 us, 2110 with the two products on shared columns.  What a task
// adds to its product is brought by bulk copies too: read by the rows' own threads it took 7000 clocks of a task, 32 lines an instruction.
// Bound, where X is large, by these copies: a step takes about 1250 clocks, its MMAs 768, and 52 bytes a clock come from L2 to each SM.
// Two 2048 x 8192 in bf16: MMAs busy 58 % of 1.77 ms.  Where X is small, by the chain of products: 512 x 4608 in fp32 (190 us) is fifteen of them one
// after the other, each waiting for the last one's results (about 1 us from its last MMA to the next one's first tile) and its own sums.
// hi hi is summed apart from the other two products: the tensor core's sums drift towards zero
// with their length, and those of small numbers do not notice.  For the same reason a long sum is cut: the epilogue adds the
// pieces up in registers, in fp32 with rounding.  Pieces are of 256 k for fp32 results (512 x 4608: error 1.1e-6; 2e-6 with 512, 3e-6 with 1024,
// 1 to 2 % faster each) and of 1024 k where the result is rounded to 16 bits or is a small part of a weight.
//
// Order.  Tasks are numbered product by product, those of all matrices together, and taken one by one off a counter.  A task waits until its
// matrix's earlier tasks are done, which a counter of the matrix tells.  What it waits for has a lower number, so it has been taken by a CTA
// that runs: however few CTAs run at a time, one of them can go on.
constexpr int kOThreads = 320;
constexpr int kOSlots = 5;                                 // of two tiles: hi and lo of an operand of a step
constexpr int kORing = 4;                                  // tasks between the warps
constexpr uint32_t kOSlot = 2 * kOrthoTile;
constexpr uint32_t kOStaging = 8 * 8192;                   // an epilogue warp's 32 rows x 64 columns, hi and lo, or fp32

struct OrthoCtl {
    uint64_t full[kOSlots], empty[kOSlots], acc_full[2], acc_empty[2], ring_full[kORing], ring_empty[kORing], old_full[8];
    int ring[kORing];
    uint32_t tmem_base;
    int abort_flag;
};

// An operand's tiles: steps below `turn` are whole tiles side by side from `rows` on, the k along them (K-major); the others halves of
// two tiles, the k down them (MN-major), from `cols` on.
struct OrthoOperand {
    long long rows, cols, pitch, lo;           // pitch: of a row of tiles; lo: from hi to lo
    int turn;
};

struct OrthoTask {
    const OrthoItem *it;
    uint8_t *m;                  // the matrix's part of the workspace
    int op, x, q;                // which product; X's and Q's places before it
    bool update, last;           // of X's size; the last product
    int phase, copy;
    bool narrow;                 // 64 columns
    int i, j;                    // row and column of the tile of 128 x 128 (or 64)
    int lower;                   // its number in the lower half
    int split;                   // piece of its k (A = X X^T)
    int from, to;                // steps of k
};

__device__ __forceinline__ OrthoTask ortho_task(const OrthoTable &tab, uint8_t *ws, int t) {
    OrthoTask k;
    int lo = 0, hi = tab.phases - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.first[mid] <= t) lo = mid; else hi = mid - 1;
    }
    k.phase = lo;
    t -= tab.first[lo];
    const int word = tab.op[lo];
    k.op = word & kOrthoOpMask;
    k.x = word & kOrthoX ? 1 : 0;
    k.q = word & kOrthoQSource ? 1 : 0;
    k.last = word & kOrthoLast;
    k.update = k.op >= kOrthoUpdate;
    const int op = k.op;
    k.narrow = tab.narrow && !k.update;
    const int squares = (op == kOrthoBQ ? 2 : 1) << tab.narrow;
    auto first = [op, squares](const OrthoItem &i) {
        return op >= kOrthoUpdate ? i.first_update : op == kOrthoGram ? i.first_gram : squares * i.first_square;
    };
    k.it = &tab.item[find_item(tab, t, first)];
    const OrthoItem &it = *k.it;
    const int side = min(it.rows, it.cols);
    int local = t - first(it);
    k.split = k.lower = 0;
    if (k.update) {
        const int per = it.rt * it.ct;
        k.copy = local / per;
        local -= k.copy * per;
        k.i = local / it.ct;
        k.j = local - k.i * it.ct;
    } else {
        const int per = ortho_lower(it.rt, it.ct) << tab.narrow;
        if (op == kOrthoGram) {
            const int whole = local / it.splits;
            k.split = local - whole * it.splits;
            local = whole;
        } else if (op == kOrthoBQ) {               // a matrix's tiles of B, then those of Q
            const int both = local / per;
            k.op = both & 1 ? kOrthoQ : kOrthoB;
            local -= both * per - (both >> 1) * per;
        }
        k.copy = local / per;
        local -= k.copy * per;
        k.lower = local;
        // row i of the lower half starts at i (i + 1) / 2, twice that where tiles are narrow
        const int pair = local >> tab.narrow;
        int i = (int)((sqrtf(8.f * (float)pair + 1.f) - 1.f) * 0.5f);
        while (i * (i + 1) / 2 > pair) --i;
        while ((i + 1) * (i + 2) / 2 <= pair) ++i;
        k.i = i;
        k.j = local - ((i * (i + 1) / 2) << tab.narrow);
    }
    k.m = ws + it.base + k.copy * it.bytes;
    k.from = op == kOrthoGram ? k.split * it.per_split : 0;
    k.to = ((op == kOrthoGram ? max(it.rows, it.cols) : side) + 63) / 64;
    if (op == kOrthoGram) k.to = min(k.to, k.from + it.per_split);
    return k;
}

// block: of 128 rows, or, narrow, of 64.  turn: never, 0 (always) or -1: where the symmetric matrix's upper half begins
__device__ __forceinline__ OrthoOperand ortho_operand(long long at, int tiles, int block, bool narrow, int turn, long long lo) {
    const long long pitch = 2LL * tiles * kOrthoTile;
    if (!narrow) return {at + block * pitch, at + 2LL * block * kOrthoTile, pitch, lo, turn < 0 ? 2 * (block + 1) : turn};
    return {at + (block >> 1) * pitch + (block & 1) * (kOrthoTile / 2), at + (long long)block * kOrthoTile, pitch, lo,
            turn < 0 ? 2 * ((block >> 1) + 1) : turn};
}
__device__ __forceinline__ void ortho_operands(const OrthoTask &k, OrthoOperand &a, OrthoOperand &b) {
    const OrthoItem &it = *k.it;
    const OrthoPlace place(it.rt, it.ct);
    const int d = min(it.rt, it.ct), never = 1 << 24;           // (a matrix has less than 2^23 tiles of two steps)
    const bool tall = it.rows > it.cols;
    const long long x = place.x(k.x);
    if (k.op == kOrthoGram) {
        a = ortho_operand(x, it.ct, k.i, false, tall ? 0 : never, place.x_bytes);
        b = ortho_operand(x, it.ct, k.j, k.narrow, tall ? 0 : never, place.x_bytes);
    } else if (!k.update) {
        const bool square = k.op == kOrthoSquare || k.op == kOrthoSquareQ;
        const long long left = square ? place.a() : place.r();
        const long long right = square || k.op == kOrthoB ? place.a() : k.op == kOrthoA ? place.b() : place.q(k.q);
        a = ortho_operand(left, d, k.i, false, -1, place.s_bytes);
        b = ortho_operand(right, d, k.j, k.narrow, -1, place.s_bytes);
    } else {
        const long long by = k.op == kOrthoUpdate ? place.r() : place.q(k.q);
        if (tall) {
            a = ortho_operand(x, it.ct, k.i, false, never, place.x_bytes);
            b = ortho_operand(by, d, k.j, false, -1, place.s_bytes);
        } else {
            a = ortho_operand(by, d, k.i, false, -1, place.s_bytes);
            b = ortho_operand(x, it.ct, k.j, false, 0, place.x_bytes);
        }
    }
}

// Where the next step's hi lies; lo behind it.
struct OrthoCursor {
    const uint8_t *p, *cols;
    long long pitch, lo;
    int turn;
    __device__ __forceinline__ OrthoCursor(const uint8_t *m, const OrthoOperand &o, int s)
        : cols(m + o.cols + (o.turn >> 1) * o.pitch), pitch(o.pitch), lo(o.lo), turn(o.turn) {          // (turn is even)
        p = s < turn ? m + o.rows + (long long)s * kOrthoTile : m + o.cols + (s >> 1) * pitch + (s & 1) * (kOrthoTile / 2);
    }
    __device__ __forceinline__ void next(int s) {
        ++s;
        if (s < turn) p += kOrthoTile;
        else if (s == turn) p = cols;
        else p += s & 1 ? (long long)(kOrthoTile / 2) : pitch - kOrthoTile / 2;
    }
};

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

__device__ __forceinline__ int load_acquire(const int *p) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void add_release(int *p, int v) { asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory"); }
// Between ordinary accesses to global memory and those of bulk copies.
__device__ __forceinline__ void fence_proxy_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

template <class T>
__global__ void __launch_bounds__(kOThreads, 1) ortho_product_kernel(const __grid_constant__ OrthoTable tab, uint8_t *__restrict__ ws, int *err) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *staging = tiles + kOSlots * kOSlot;
    OrthoCtl *ctl = (OrthoCtl *)(staging + kOStaging);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &ctl->abort_flag;
    int *taken = (int *)ws, *done = taken + 1, *tickets = done + tab.matrices;
    auto give_up = [&]() { atomicOr(err, ERRW_TIMEOUT); ctl->abort_flag = 1; };

    if (threadIdx.x == 64) {
        for (int s = 0; s < kOSlots; ++s) { mbar_init(&ctl->full[s], 1); mbar_init(&ctl->empty[s], 1); }
        for (int w = 0; w < 8; ++w) mbar_init(&ctl->old_full[w], 1);
        for (int a = 0; a < 2; ++a) { mbar_init(&ctl->acc_full[a], 1); mbar_init(&ctl->acc_empty[a], 8); }
        for (int r = 0; r < kORing; ++r) { mbar_init(&ctl->ring_full[r], 1); mbar_init(&ctl->ring_empty[r], 9); }
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
            const int total = tab.first[tab.phases];
            uint32_t it = 0, n = 0;
            bool ok = true;
            // (issuing loops step addresses: what they form anew each step, they form at the price of a step's copies)
            const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]), tiles0 = smem_u32(tiles);
            uint32_t slot = 0, ph = 1;
            bool free = false;
            for (;; ++n) {
                // (taken when its loads can begin: a task held in advance waits here while other CTAs have nothing to do)
                const int t = atomicAdd(taken, 1);
                const uint32_t r = n % kORing;
                ok = mbar_wait_bounded(&ctl->ring_empty[r], ((n / kORing) & 1u) ^ 1u, abort_flag);
                if (!ok) break;
                if (t >= total) {
                    ctl->ring[r] = -1;
                    mbar_arrive(&ctl->ring_full[r]);
                    break;
                }
                const OrthoTask k = ortho_task(tab, ws, t);
                // the eight warps' shares of every earlier task of the matrix
                const int need = 8 * (tab.lowers[k.phase] * ortho_lower(k.it->rt, k.it->ct) + tab.xs[k.phase] * k.it->rt * k.it->ct);
                const int *flag = done + k.it->first_matrix + k.copy;
                if (load_acquire(flag) < need) {
                    const uint64_t t0 = globaltimer_ns();
                    uint32_t spins = 0;
                    while (load_acquire(flag) < need) {
                        __nanosleep(20);
                        if ((++spins & 255u) == 0 && (*abort_flag || globaltimer_ns() - t0 > 2000000000ull)) { ok = false; break; }
                    }
                    if (!ok) break;
                }
                fence_proxy_async_global();
                ctl->ring[r] = t;
                mbar_arrive(&ctl->ring_full[r]);
                OrthoOperand a, b;
                ortho_operands(k, a, b);
                OrthoCursor at[2] = {OrthoCursor(k.m, a, k.from), OrthoCursor(k.m, b, k.from)};
                for (int s = k.from; ok && s < k.to; ++s)
#pragma unroll
                    for (int part = 0; part < 2; ++part, ++it) {
                        if (!free) ok = ok && mbar_wait_bounded(empty0 + slot * 8, ph, abort_flag);
                        if (!ok) break;
                        const uint32_t bar = full0 + slot * 8, dst = tiles0 + slot * kOSlot;
                        if (++slot == kOSlots) { slot = 0; ph ^= 1u; }
                        free = mbar_test_wait(empty0 + slot * 8, ph);
                        const bool narrow = part && k.narrow;
                        const uint32_t bytes = narrow ? kOrthoTile / 2 : kOrthoTile;
                        mbar_arrive_expect_tx(bar, 2 * bytes);
                        OrthoCursor &c = at[part];
                        if (s < c.turn || narrow) {
                            const uint32_t one = s < c.turn ? bytes : kOrthoTile / 2;
                            bulk_load(dst, c.p, one, bar);
                            bulk_load(dst + bytes, c.p + c.lo, one, bar);
                        } else {
                            bulk_load(dst, c.p, kOrthoTile / 2, bar);
                            bulk_load(dst + kOrthoTile / 2, c.p + kOrthoTile, kOrthoTile / 2, bar);
                            bulk_load(dst + kOrthoTile, c.p + c.lo, kOrthoTile / 2, bar);
                            bulk_load(dst + 3 * kOrthoTile / 2, c.p + c.lo + kOrthoTile, kOrthoTile / 2, bar);
                        }
                        c.next(s);
                    }
                if (!ok) break;
            }
            if (!ok) {
                give_up();
                for (uint32_t j = it > kOSlots ? it - kOSlots : 0; j < it; ++j)          // let the copies in flight land
                    mbar_wait_bounded(&ctl->full[j % kOSlots], (j / kOSlots) & 1u, nullptr, 200000000ull);
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t hi = smem_desc_hi_sw128(1024), segment_mask = (uint32_t)tab.segment_mask;
            const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]), tiles_lo = smem_u32(tiles) >> 4;
            uint32_t slot = 0, ph = 0, acc_it = 0;
            bool ok = true;
            for (uint32_t n = 0;; ++n) {
                const uint32_t r = n % kORing;
                ok = mbar_wait_bounded(&ctl->ring_full[r], (n / kORing) & 1u, abort_flag, 4000000000ull);
                if (!ok) break;
                const int t = ctl->ring[r];
                mbar_arrive(&ctl->ring_empty[r]);
                if (t < 0) break;
                const OrthoTask k = ortho_task(tab, ws, t);
                OrthoOperand a, b;
                ortho_operands(k, a, b);
                const uint32_t one0 = idesc_h16_f32(128, k.narrow ? 64 : 128, 0, 0, 1), b_lo = kOrthoTile >> 4;
                for (int s = k.from; s < k.to; ++s) {
                    const uint32_t acc = acc_it & 1u, d = tmem_base + acc * 256u, first = (uint32_t)(s - k.from) & segment_mask;
                    if (first == 0) {
                        ok = mbar_wait_bounded(&ctl->acc_empty[acc], ((acc_it >> 1) & 1u) ^ 1u, abort_flag);
                        if (!ok) break;
                        tc_fence_after_sync();
                    }
                    // bit 15 of the instruction's descriptor: A MN-major, 16: B; the leading byte offset is 8192 then, else 16
                    const uint32_t a_mn = s >= a.turn, b_mn = s >= b.turn, major = a_mn << 15 | b_mn << 16;
                    const uint32_t sa = a_mn ? 128u : 2u, sb = b_mn ? 128u : 2u;
                    ok = mbar_wait_bounded(full0 + slot * 8, ph, abort_flag);
                    if (!ok) break;
                    const uint32_t a_hi = tiles_lo + slot * (kOSlot >> 4) + (a_mn ? 512u << 16 : 1u << 16), a_lo = a_hi + (kOrthoTile >> 4);
                    const uint32_t done_a = empty0 + slot * 8;
                    if (++slot == kOSlots) { slot = 0; ph ^= 1u; }
                    ok = mbar_wait_bounded(full0 + slot * 8, ph, abort_flag);
                    if (!ok) break;
                    const uint32_t b_hi = tiles_lo + slot * (kOSlot >> 4) + (b_mn ? 512u << 16 : 1u << 16), done_b = empty0 + slot * 8;
                    if (++slot == kOSlots) { slot = 0; ph ^= 1u; }
                    if (k.narrow) {
                        const uint32_t both = idesc_h16_f32(128, 128, 0, 0, 1) | major, one = one0 | major;
#pragma unroll
                        for (uint32_t q = 0; q < 4; ++q) {
                            umma_bf16_ss_sel(d, a_hi + q * sa, hi, b_hi + q * sb, hi, both, first + q);
                            umma_bf16_ss_sel(d + 128, a_lo + q * sa, hi, b_hi + q * sb, hi, one, first + q);
                        }
                    } else {
                        const uint32_t one = one0 | major;
#pragma unroll
                        for (uint32_t q = 0; q < 4; ++q) {
                            umma_bf16_ss_sel(d, a_hi + q * sa, hi, b_hi + q * sb, hi, one, first + q);
                            umma_bf16_ss_sel(d + 128, a_hi + q * sa, hi, b_hi + b_lo + q * sb, hi, one, first + q);
                            umma_bf16_ss_halves<true>(d + 128, a_lo + q * sa, hi, b_hi + q * sb, hi, one);
                        }
                    }
                    umma_commit(done_a);
                    umma_commit(done_b);
                    if (s + 1 == k.to || first == segment_mask) { umma_commit(&ctl->acc_full[acc]); ++acc_it; }
                }
                if (!ok) break;
            }
            if (!ok) give_up();
        }
    } else {
        // A warp has 32 rows of 64 columns: a quarter of a tile of the workspace, 4 KB side by side there.
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        uint8_t *buf = staging + (warp - 2) * 8192;
        const uint32_t row = quarter * 32 + lane;
        const int segment_shift = __popc(tab.segment_mask);
        uint32_t acc_it = 0, old_ph = 0;
        bool ok = true;
        for (uint32_t n = 0;; ++n) {
            const uint32_t r = n % kORing;
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->ring_full[r], (n / kORing) & 1u, abort_flag, 4000000000ull));
            if (!ok) break;
            const int t = ctl->ring[r];
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl->ring_empty[r]);
            if (t < 0) break;
            const OrthoTask k = ortho_task(tab, ws, t);
            const OrthoItem &it = *k.it;
            const OrthoPlace place(it.rt, it.ct);
            const int segments = (k.to - k.from + tab.segment_mask) >> segment_shift;
            if (k.narrow && half) {                             // (64 columns are four warps' work)
                for (int g = 0; g < segments; ++g, ++acc_it) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->acc_full[acc_it & 1u], (acc_it >> 1) & 1u, abort_flag));
                    if (!ok) break;
                    if (lane == 0) mbar_arrive(&ctl->acc_empty[acc_it & 1u]);
                }
                if (!ok) break;
                continue;
            }
            // numbers are 2^10 times what they stand for (Q's 2^8), sums of products 2^20 times (2^18)
            const long long x_at = ((long long)k.i * 2 * it.ct + 2 * k.j + half) * kOrthoTile;
            const long long s_at = ((long long)k.i * 2 * min(it.rt, it.ct) + (k.narrow ? k.j : 2 * k.j + half)) * kOrthoTile;
            const long long lo_at = k.update ? place.x_bytes : place.s_bytes;
            long long old_at = -1, to_at;
            float v[64], f_old = kOrthoCoefA, f_new = 1.f / kOrthoScale;
            switch (k.op) {
                case kOrthoGram: to_at = place.a() + s_at; break;
                case kOrthoSquare: case kOrthoSquareQ:
                    old_at = place.a() + s_at; to_at = place.r() + s_at; f_old = kOrthoCoefB; f_new = kOrthoCoefC / kOrthoScale; break;
                case kOrthoB: old_at = place.a() + s_at; to_at = place.b() + s_at; break;
                case kOrthoA: old_at = place.b() + s_at; to_at = place.a() + s_at; break;
                case kOrthoQ: old_at = place.q(k.q) + s_at; to_at = place.q(k.q ^ 1) + s_at; break;
                case kOrthoUpdate: old_at = place.x(k.x) + x_at; to_at = place.x(k.x ^ 1) + x_at; break;
                default: to_at = place.x(k.x ^ 1) + x_at; f_new = 1.f / kOrthoQScale; break;
            }
            if (old_at < 0) {
#pragma unroll
                for (int i = 0; i < 64; ++i) v[i] = 0.f;
            } else {
                const uint8_t *old = k.m + old_at + quarter * 4096;
                if (lane == 0) {
                    fence_proxy_async_global();                 // (the producer saw the counter)
                    fence_proxy_async_smem();
                    const uint32_t bar = smem_u32(&ctl->old_full[warp - 2]);
                    mbar_arrive_expect_tx(bar, 8192);
                    bulk_load(smem_u32(buf), old, 4096, bar);
                    bulk_load(smem_u32(buf) + 4096, old + lo_at, 4096, bar);
                }
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->old_full[warp - 2], old_ph, abort_flag));
                if (!ok) {                                      // (the copy in flight lands before the block ends)
                    if (lane == 0) mbar_wait_bounded(&ctl->old_full[warp - 2], old_ph, nullptr, 200000000ull);
                    __syncwarp();
                    break;
                }
                old_ph ^= 1u;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint4 oh = *(const uint4 *)(buf + ortho_chunk(lane, c)), ol = *(const uint4 *)(buf + 4096 + ortho_chunk(lane, c));
                    const float2 o[4] = {half_pair(oh.x, ol.x), half_pair(oh.y, ol.y), half_pair(oh.z, ol.z), half_pair(oh.w, ol.w)};
#pragma unroll
                    for (int e = 0; e < 4; ++e) { v[8 * c + 2 * e] = f_old * o[e].x; v[8 * c + 2 * e + 1] = f_old * o[e].y; }
                }
            }
            for (int g = 0; g < segments; ++g, ++acc_it) {
                const uint32_t acc = acc_it & 1u;
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->acc_full[acc], (acc_it >> 1) & 1u, abort_flag));
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t from = tmem_base + acc * 256u + half * 64u + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t p[32], q[32];
                    tmem_ld_32x32(from + (k.narrow ? 64 : 0) + h * 32, p);
                    tmem_ld_32x32(from + 128 + h * 32, q);
                    tmem_ld_wait();
                    if (k.narrow) {                             // hi hi | hi lo | lo hi
#pragma unroll
                        for (int i = 0; i < 32; ++i) q[i] = __float_as_uint(__uint_as_float(p[i]) + __uint_as_float(q[i]));
                        tmem_ld_32x32(from + h * 32, p);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[h * 32 + i] = fmaf(f_new, __uint_as_float(p[i]) + __uint_as_float(q[i]), v[h * 32 + i]);
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->acc_empty[acc]);
            }
            if (!ok) break;
            if (k.op == kOrthoGram && it.splits > 1) {
                // The piece goes to memory, [4 columns][row] by chunks of 16 bytes; the warp whose piece is the last of this share of the
                // tile adds all of them up, in their order.
                const int part_bytes = k.narrow ? 32768 : 65536;
                float4 *part = (float4 *)(k.m + place.parts(it.wide) + ((long long)k.lower * it.splits + k.split) * part_bytes) + half * 2048 + row;
#pragma unroll
                for (int c = 0; c < 16; ++c) __stcg(part + c * 128, make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]));
                __threadfence();
                __syncwarp();
                int ticket = 0;
                if (lane == 0)
                    ticket = atomicAdd(tickets + 8 * (it.first_square + k.copy * ortho_lower(it.rt, it.ct)) + (k.narrow ? 4 : 8) * k.lower + (warp - 2), 1);
                ticket = __shfl_sync(0xffffffffu, ticket, 0);
                if ((ticket + 1) % it.splits != 0) continue;
                __threadfence();
                part -= (long long)k.split * (part_bytes / 16);
#pragma unroll
                for (int i = 0; i < 64; ++i) v[i] = 0.f;
                for (int p = 0; p < it.splits; ++p) {
                    float4 f[16];
#pragma unroll
                    for (int c = 0; c < 16; ++c) f[c] = __ldcg(part + (long long)p * (part_bytes / 16) + c * 128);
#pragma unroll
                    for (int c = 0; c < 16; ++c) { v[4 * c] += f[c].x; v[4 * c + 1] += f[c].y; v[4 * c + 2] += f[c].z; v[4 * c + 3] += f[c].w; }
                }
            }
            if (!k.last) {
                // through the warp's staging, where its share of a tile lies as it does in memory
                auto put = [&](uint8_t *to) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        uint32_t wh[4], wl[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const __half2 h = __floats2half2_rn(v[8 * c + 2 * e], v[8 * c + 2 * e + 1]);
                            const float2 back = __half22float2(h);
                            const __half2 l = __floats2half2_rn(v[8 * c + 2 * e] - back.x, v[8 * c + 2 * e + 1] - back.y);
                            wh[e] = *reinterpret_cast<const uint32_t *>(&h);
                            wl[e] = *reinterpret_cast<const uint32_t *>(&l);
                        }
                        *(uint4 *)(buf + ortho_chunk(lane, c)) = make_uint4(wh[0], wh[1], wh[2], wh[3]);      // (its rows start on a multiple of 8)
                        *(uint4 *)(buf + 4096 + ortho_chunk(lane, c)) = make_uint4(wl[0], wl[1], wl[2], wl[3]);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        bulk_store(to, buf, 4096);
                        bulk_store(to + lo_at, buf + 4096, 4096);
                        tma_store_commit();
                    }
                };
                put(k.m + to_at + quarter * 4096);
                if (k.op == kOrthoSquareQ) {
                    const int diagonal = (k.narrow ? k.j >> 1 : k.j) == k.i ? (int)row - (k.narrow ? k.j & 1 : half) * 64 : -1;
#pragma unroll
                    for (int i = 0; i < 64; ++i) v[i] = v[i] * (kOrthoQScale / kOrthoScale) + (i == diagonal ? kOrthoCoefA * kOrthoQScale : 0.f);
                    if (lane == 0) tma_store_wait_read<0>();
                    __syncwarp();
                    put(k.m + place.q(0) + s_at + quarter * 4096);
                }
                if (lane == 0) {
                    tma_store_wait_all<0>();                    // (written, and seen by this thread, whose release passes that on)
                    add_release(done + it.first_matrix + k.copy, 1);
                }
                __syncwarp();
            } else {
                // through the staging, chunks of four in an order that spreads a column over the banks, then row by row
                const int r0 = k.i * 128 + quarter * 32, rows = min(32, it.rows - r0);
                const long long base = k.copy * ((long long)it.rows * it.cols) + (long long)r0 * it.cols;
#pragma unroll
                for (int c = 0; c < 16; ++c)
                    *(float4 *)(buf + lane * 256 + ((c ^ (lane & 15)) << 4)) = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
                __syncwarp();
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int c = k.j * 128 + half * 64 + h * 32 + lane;
                    if (c >= it.cols) continue;
                    auto at = [&](int i) { return *(const float *)(buf + i * 256 + (((h * 8 + (lane >> 2)) ^ (i & 15)) << 4) + (lane & 3) * 4) * (1.f / kOrthoScale); };
                    T *out = (T *)it.out;
                    if (tab.muon) {
                        float *master = it.master + base + c;
                        for (int i0 = 0; i0 < rows; i0 += 16) {
                            float w[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) w[i] = i0 + i < rows ? master[(long long)(i0 + i) * it.cols] : 0.f;
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (i0 + i < rows) {
                                    const float x = fmaf(-it.scale, at(i0 + i), tab.keep * w[i]);
                                    master[(long long)(i0 + i) * it.cols] = x;
                                    if (out) out[base + (long long)(i0 + i) * it.cols + c] = from_f32<T>(x);
                                }
                        }
                    } else {
                        for (int i = 0; i < rows; ++i) out[base + (long long)i * it.cols + c] = from_f32<T>(at(i));
                    }
                }
                __syncwarp();
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
    constexpr int smem = 1024 + kOSlots * kOSlot + kOStaging + sizeof(OrthoCtl);
    if (e = max_dynamic_smem_once(kernel, smem, &attr); e != cudaSuccess) return e;
    prefer_max_shared_once(kernel, &carve);
    const int sms = device_sm_count(), widest = t.updates > t.grams ? t.updates : t.grams;
    return launch_pdl(kernel, dim3((unsigned)(widest < sms ? widest : sms)), dim3(kOThreads), smem, st, t, ws, err);
}

}  // namespace

// Two steps at a time or more save 9 m^2 (n - m) operations of five steps', and cost two more products in the chain: they pay where X is long, so that the
// chain is of shorter products, and where there is much to save.  us in bf16, directly and so: 512 x 4608 199 and 179, 256 x 1152 138 and 130, 512 x 1536
// 164 and 163, 1000 x 2048 248 and 251, 512 x 768 154 and 158; 2048 x 2560 695 and 627, three of 1956 x 3501 2131 and 1787, two of 988 x 1865
// (saved / 9: 1.7e9) 380 and 349, 1024 x 2048 (1.1e9) 290 and 294.
// In a list the heaviest matrix says whether X is long: 640 x 640, 700 x 640 and 5 x 1 take 176 us directly, 187 where 5 x 1 says it.
void OrthoChoice::add(int rows, int cols, int count) {
    const double m = std::min(rows, cols), n = std::max(rows, cols);
    const double work = m * m * (3. * n + m) * count;
    if (work > heaviest) {                         // (whose chain the others of the list run beside)
        heaviest = work;
        longer = n >= 2.5 * m;
    }
    saved += m * m * (n - m) * count;
}
bool OrthoChoice::wide() const { return longer || saved > 1.3e9; }

static void ortho_phases(OrthoTable &t, bool wide) {
    int x = 0, lowers = 0, xs = 0, at = 0, n = 0;
    auto add = [&](int op, int q = 0) {
        const bool update = op >= kOrthoUpdate;
        t.op[n] = (uint16_t)(op | (x ? kOrthoX : 0) | (q ? kOrthoQSource : 0));
        t.lowers[n] = (uint16_t)lowers;
        t.xs[n] = (uint16_t)xs;
        t.first[n++] = at;
        at += update ? t.updates : op == kOrthoGram ? t.grams : t.squares << (t.narrow + (op == kOrthoBQ));
        if (update) { ++xs; x ^= 1; } else lowers += op == kOrthoBQ ? 2 : 1;
    };
    const int stages = wide ? (t.steps + 2) / 3 : t.steps;
    for (int s = 0, left = t.steps; s < stages; ++s) {
        const int k = (left + stages - s - 1) / (stages - s);          // 5: 3 and 2
        left -= k;
        add(kOrthoGram);
        if (k == 1) {
            add(kOrthoSquare);
            add(kOrthoUpdate);
            continue;
        }
        int q = 0;
        for (int i = 0; i < k; ++i) {
            add(i ? kOrthoSquare : kOrthoSquareQ);
            if (i + 1 < k) {
                add(i ? kOrthoBQ : kOrthoB, q);
                add(kOrthoA);
            } else {
                add(kOrthoQ, q);
            }
            if (i) q ^= 1;
        }
        add(kOrthoUpdateQ, q);
    }
    t.op[n - 1] |= kOrthoLast;
    t.first[n] = at;
    t.phases = n;
}

size_t ortho_plan(OrthoTable &t, bool wide) {
    const int sms = device_sm_count();
    t.sums = t.tiles = t.grams = t.squares = t.updates = t.matrices = 0;
    for (int i = 0; i < t.items; ++i) {
        OrthoItem &it = t.item[i];
        it.wide = wide;
        it.rt = (it.rows + 127) / 128;
        it.ct = (it.cols + 127) / 128;
        it.first_sum = t.sums; it.first_tile = t.tiles; it.first_square = t.squares; it.first_update = t.updates; it.first_matrix = t.matrices;
        t.sums += it.count * ortho_chunks(it);
        t.tiles += it.count * it.rt * it.ct * 2;
        t.squares += it.count * ortho_lower(it.rt, it.ct);
        t.updates += it.count * it.rt * it.ct;
        t.matrices += it.count;
    }
    // Where A's tiles leave half the SMs idle, they are halved: a step's copies, which come at some 52 bytes a clock, are what a product waits for
    // (a step of 128 x 128 takes 1250 clocks, of 128 x 64 930).  Where they still leave SMs idle, A's sums are cut: a step takes 0.4 us, adding
    // up a piece 0.7 us.
    t.narrow = 2 * t.squares <= sms;
    const int tiles_of_a = t.squares << t.narrow;
    for (int i = 0; i < t.items; ++i) {
        OrthoItem &it = t.item[i];
        const int steps = ((it.rows > it.cols ? it.rows : it.cols) + 63) / 64;
        int pieces = 1;
        while ((pieces + 1) * (pieces + 1) * 5 <= steps * 2) ++pieces;
        if (pieces > sms / tiles_of_a) pieces = sms / tiles_of_a;
        if (pieces < 1) pieces = 1;
        it.per_split = (steps + pieces - 1) / pieces;
        it.splits = (steps + it.per_split - 1) / it.per_split;
        it.first_gram = t.grams;
        t.grams += it.count * (ortho_lower(it.rt, it.ct) << t.narrow) * it.splits;
    }
    ortho_phases(t, wide);
    long long end = (long long)align_up((size_t)ortho_words(t) * sizeof(int), 1024);
    for (int i = 0; i < t.items; ++i) {
        OrthoItem &it = t.item[i];
        it.base = end;
        it.bytes = ortho_sums_at(it) + (long long)align_up((size_t)ortho_chunks(it) * sizeof(double), 1024);
        end += it.count * it.bytes;
    }
    return (size_t)end;
}

cudaError_t launch_ortho(const OrthoTable &t, void *workspace, cudaStream_t st) {
    if (ortho_small_pays(t)) return launch_ortho_small(t, st);
    switch (t.dtype) {
        case CONVBN_F32: return launch_ortho_t<float>(t, (uint8_t *)workspace, st);
        case CONVBN_F16: return launch_ortho_t<__half>(t, (uint8_t *)workspace, st);
        default: return launch_ortho_t<__nv_bfloat16>(t, (uint8_t *)workspace, st);
    }
}

}  // namespace convbn
