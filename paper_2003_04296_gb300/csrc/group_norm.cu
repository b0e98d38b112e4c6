// group_norm.cu -- forward of the group norm with an activation on
// channels-last rows (group_norm.cuh: statistics, tiles and plans).
#include "group_norm.cuh"

namespace minw {
namespace gn {

// ---------------------------------------------------------------------------
// Groups wider than a block's lanes: statistics per chunk and channel, merged
// per group, then a second pass over x.
// ---------------------------------------------------------------------------

template <typename T, int V>
__global__ void __launch_bounds__(THREADS, 4) stat_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int NP = (V + 1) / 2;
    __shared__ float2 red[THREADS * V];
    const Place w = place<V>(a, blockIdx.x);
    Pair m[NP], q[NP];
    channel_stats<T, V, V == 1 ? 16 : 4>(
        static_cast<const T *>(a.x) + ((int64_t)w.b * a.P + w.p0 + w.row) * a.ldx + w.c, w.rows * a.ldx, w.n, m, q);
    // rows of the block: the first `more` hold `most` pixels each, the others one fewer
    const int W = a.L * V, np = w.p1 - w.p0, whole = (np - 1) / w.rows;
    const int more = np - whole * w.rows;
    const float most = (float)(whole + 1);
    if (w.row < w.rows) {
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const float2 mk = halves(m[k]), qk = halves(q[k]);
            red[w.row * W + w.lane * V + 2 * k] = make_float2(mk.x, qk.x);
            if (V > 1) red[w.row * W + w.lane * V + 2 * k + 1] = make_float2(mk.y, qk.y);
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < W; e += THREADS) {
        const int c = w.slab * W + e;
        if (c >= a.C) break;
        float s = 0.0f;
        for (int r = 0; r < w.rows; ++r) s = fmaf(r < more ? most : most - 1.0f, red[r * W + e].x, s);
        const float mean = s / (float)np;
        float M2 = 0.0f;
        for (int r = 0; r < w.rows; ++r) {
            const float2 t = red[r * W + e];
            const float d = t.x - mean;
            M2 += fmaf(d * d, r < more ? most : most - 1.0f, t.y);
        }
        a.part[((int64_t)w.b * a.chunks + w.chunk) * a.C + c] = make_float2(mean, M2);
    }
}

// Block = one image's group: merges its chunks x channels.
__global__ void __launch_bounds__(THREADS) stat_merge_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    __shared__ float red[THREADS / 32];
    const int b = (int)(blockIdx.x / a.G), g = (int)(blockIdx.x % a.G);
    const int entries = a.chunks * a.Cg;
    const float2 *part = a.part + (int64_t)b * a.chunks * a.C + g * a.Cg;
    auto block_sum = [&](float v) {
        v = warp_sum(v);
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < THREADS / 32; ++k) s += red[k];
        __syncthreads();
        return s;
    };
    const float n = (float)a.P * (float)a.Cg;
    float s = 0.0f;
#pragma unroll 4
    for (int e = threadIdx.x; e < entries; e += THREADS) {
        const int k = e / a.Cg;
        s = fmaf((float)(min(a.P, (k + 1) * a.ppc) - k * a.ppc), part[(int64_t)k * a.C + e % a.Cg].x, s);
    }
    const float mean = block_sum(s) / n;
    s = 0.0f;
#pragma unroll 4
    for (int e = threadIdx.x; e < entries; e += THREADS) {
        const int k = e / a.Cg;
        const float2 t = part[(int64_t)k * a.C + e % a.Cg];
        const float d = t.x - mean;
        s += fmaf(d * d, (float)(min(a.P, (k + 1) * a.ppc) - k * a.ppc), t.y);
    }
    const float rstd = rsqrtf(block_sum(s) / n + a.eps);
    if (threadIdx.x == 0) {
        a.stat[blockIdx.x] = make_float2(mean, rstd);
        if (a.mean) a.mean[blockIdx.x] = mean;
        if (a.rstd) a.rstd[blockIdx.x] = rstd;
    }
}

template <typename T, typename TY, int V>
__global__ void __launch_bounds__(THREADS, 4) apply_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int NP = (V + 1) / 2;
    const Place w = place<V>(a, (int64_t)gridDim.x - 1 - blockIdx.x);     // the last chunks read are still in L2
    if (w.n == 0) return;
    Pair nm[NP], sc[NP], sh[NP];
    {
        float ga[V], be[V], mean[V];
        load_affine<V>(a, w.c, ga, be);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float2 t = a.stat[(int64_t)w.b * a.G + (w.c + i) / a.Cg];
            mean[i] = -t.x;
            ga[i] *= t.y;
        }
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            nm[k] = pick<V>(mean, k);
            sc[k] = pick<V>(ga, k);
            sh[k] = pick<V>(be, k);
        }
    }
    const int64_t p = (int64_t)w.b * a.P + w.p0 + w.row;
    with_act(a.act, [&](auto act) {
        apply_pixels<T, TY, V, V == 1 ? 8 : 4, act.value>(static_cast<const T *>(a.x) + p * a.ldx + w.c, w.rows * a.ldx,
                                                          static_cast<TY *>(a.y) + p * a.ldy + w.c, w.rows * a.ldy, w.n, w.n,
                                                          [](int) { return Vec<T, V>(); }, nm, sc, sh);
    });
}

// ---------------------------------------------------------------------------
// One kernel
// ---------------------------------------------------------------------------

// Sums over a block of each thread's GPT values, one per group of its channels; afterwards every thread has the
// sums of its own groups.  `per` entries (a thread's value is one) make a group, L GPT a row.
template <int GPT>
struct GroupSum {
    float part[THREADS * GPT], total[MAX_SLAB_GROUPS];
};
template <int GPT>
__device__ __forceinline__ void group_sum(float *s, GroupSum<GPT> &sm, const Args &a, const Tile &w) {
    const int lane = threadIdx.x & 31, at = a.by_per.div(w.lane * GPT);
    if (a.butterfly) {
        // lanes of a warp with the same channels, then those of a group, by exchanges; then the eight warps' sums
#pragma unroll
        for (int d = 1; d < 32; d <<= 1)
            if (d < a.per || d >= a.L) {
#pragma unroll
                for (int g = 0; g < GPT; ++g) s[g] += __shfl_xor_sync(0xffffffffu, s[g], d);
            }
        if (lane < a.L && (lane & (a.per - 1)) == 0) {
#pragma unroll
            for (int g = 0; g < GPT; ++g) sm.part[(threadIdx.x >> 5) * a.groups + at + g] = s[g];
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            s[g] = 0.0f;
#pragma unroll
            for (int k = 0; k < THREADS / 32; ++k) s[g] += sm.part[k * a.groups + at + g];
        }
    } else {
        const int row = a.L * GPT;
        if (w.row < w.rows) {
#pragma unroll
            for (int g = 0; g < GPT; ++g) sm.part[w.row * row + w.lane * GPT + g] = s[g];
        }
        __syncthreads();
        for (int g = threadIdx.x >> 5; g < a.groups; g += THREADS / 32) {      // a warp per group
            float t = 0.0f;
            for (int e = lane; e < w.rows * a.per; e += 32) {
                const int r = a.by_per.div(e);
                t += sm.part[r * row + g * a.per + e - r * a.per];
            }
            t = warp_sum(t);
            if (lane == 0) sm.total[g] = t;
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < GPT; ++g) s[g] = sm.total[a.by_per.div(w.lane * GPT + g)];
    }
}

template <int GPT>
struct Shared {
    GroupSum<GPT> sums[2];
    float2 cta[MAX_SLAB_GROUPS], all[MAX_SLAB_GROUPS];
};
static_assert(sizeof(Shared<4>) == 8 * (THREADS * 4 + MAX_SLAB_GROUPS) + 16 * MAX_SLAB_GROUPS, "plan() counts on it");

// The block's mean and M2 of each of a thread's GPT groups from its own `values` values' mean and M2 of them: the block's
// mean turns M2 into deviations from that (values (own - mean)^2 more).
template <int GPT>
__device__ __forceinline__ void merge_block(const Args &a, const Tile &w, Shared<GPT> &sm, const float *own, float values,
                                            float *mean, float *m2) {
#pragma unroll
    for (int g = 0; g < GPT; ++g) mean[g] = own[g] * values;
    group_sum<GPT>(mean, sm.sums[0], a, w);
    const float block = w.p1 > w.p0 ? __fdividef(1.0f, (float)(w.p1 - w.p0) * (float)a.Cg) : 0.0f;
#pragma unroll
    for (int g = 0; g < GPT; ++g) {
        mean[g] *= block;
        const float d = own[g] - mean[g];
        if (values > 0.0f) m2[g] = fmaf(d * d, values, m2[g]);
    }
    group_sum<GPT>(m2, sm.sums[1], a, w);
}

// The cluster's in sm.all from its blocks' (chunks first .. first + size - 1 of the image); the same sums in every block.
// Afterwards the cluster has arrived at its end (cluster_leave).
template <int GPT>
__device__ __forceinline__ void merge_cluster(const Args &a, const Tile &w, Shared<GPT> &sm, int first, int size,
                                              const float *mean, const float *m2) {
    if (w.row == 0) {
#pragma unroll
        for (int g = 0; g < GPT; ++g) sm.cta[a.by_per.div(w.lane * GPT + g)] = make_float2(mean[g], m2[g]);
    }
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    const int all = min(a.P, (first + size) * a.ppc) - min(a.P, first * a.ppc);
    const float inv = __fdividef(1.0f, (float)max(all, 1) * (float)a.Cg);
    // eight threads a group, one for each block
    for (int g = threadIdx.x >> 3; g < (a.groups + 3) / 4 * 4; g += THREADS / 8) {     // all of a warp alike
        const int k = threadIdx.x & 7;
        float2 t = make_float2(0.0f, 0.0f);
        float n = 0.0f;
        if (k < size && g < a.groups) {
            t = *cluster.map_shared_rank(&sm.cta[g], k);
            n = (float)(min(a.P, (first + k + 1) * a.ppc) - min(a.P, (first + k) * a.ppc)) * (float)a.Cg;
        }
        float s = n * t.x;
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s *= inv;
        const float d0 = t.x - s;
        float q = n > 0.0f ? fmaf(d0 * d0, n, t.y) : 0.0f;
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) q += __shfl_xor_sync(0xffffffffu, q, d);
        if (k == 0 && g < a.groups) sm.all[g] = make_float2(s, q);
    }
    cluster_done_reading();
    __syncthreads();
}

// Mean and rstd of each of a thread's groups, saved by the image's first block.
template <int GPT>
__device__ __forceinline__ void merge(const Args &a, const Tile &w, Shared<GPT> &sm, const float *own, float *m2,
                                      float values, float *mean, float *rstd) {
    merge_block<GPT>(a, w, sm, own, values, mean, m2);
    if (a.chunks > 1) {
        merge_cluster<GPT>(a, w, sm, 0, a.chunks, mean, m2);
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            const float2 t = sm.all[a.by_per.div(w.lane * GPT + g)];
            mean[g] = t.x;
            m2[g] = t.y;
        }
    }
#pragma unroll
    for (int g = 0; g < GPT; ++g) rstd[g] = rsqrtf(fmaf(m2[g], a.inv_total, a.eps));
    if (w.rank == 0 && w.row == 0) {
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            const int64_t at = (int64_t)w.b * a.G + w.slab * a.groups + a.by_per.div(w.lane * GPT + g);
            if (a.mean) a.mean[at] = mean[g];
            if (a.rstd) a.rstd[at] = rstd[g];
        }
    }
}

// Mean and M2 of a thread's groups from its channels' of n values each.
template <int V, int GPT>
__device__ __forceinline__ void fold_channels(const Pair *m, const Pair *q, int n, float *own, float *m2) {
    constexpr int W = V / GPT;
#pragma unroll
    for (int g = 0; g < GPT; ++g) {
        float f[W], s = 0.0f, d2 = 0.0f, r = 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const float2 h = halves(m[(g * W + k) / 2]), h2 = halves(q[(g * W + k) / 2]);
            f[k] = (g * W + k) % 2 ? h.y : h.x;
            s += f[k];
            r += (g * W + k) % 2 ? h2.y : h2.x;
        }
        own[g] = s * (1.0f / W);
#pragma unroll
        for (int k = 0; k < W; ++k) d2 = fmaf(f[k] - own[g], f[k] - own[g], d2);
        m2[g] = fmaf(d2, (float)n, r);
    }
}

// Minus the means, rstd gamma and beta of a thread's channels, in pairs.
template <int V, int GPT>
__device__ __forceinline__ void coefficients(const Args &a, int c, const float *mean, const float *rstd, Pair *nm, Pair *sc,
                                             Pair *sh) {
    constexpr int W = V / GPT, NP = (V + 1) / 2;
    float ga[V], be[V];
    load_affine<V>(a, c, ga, be);
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        nm[k] = pick_group<V, W>(mean, k, -1.0f);
        sc[k] = mul2(pick_group<V, W>(rstd, k), pick<V>(ga, k));
        sh[k] = pick<V>(be, k);
    }
}

// Each group's sum of a thread's sums of channel pairs: of one group, or (W = 1) of two.
template <int V, int GPT>
__device__ __forceinline__ void fold_pairs(const Pair *p, float *f) {
    constexpr int W = V / GPT;
    if constexpr (W == 1) {
#pragma unroll
        for (int k = 0; k < (V + 1) / 2; ++k) {
            const float2 h = halves(p[k]);
            f[2 * k] = h.x;
            if (V > 1) f[2 * k + 1] = h.y;
        }
    } else {
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            Pair t = p[g * W / 2];
#pragma unroll
            for (int k = 1; k < W / 2; ++k) t = add2(t, p[g * W / 2 + k]);
            const float2 h = halves(t);
            f[g] = h.x + h.y;
        }
    }
}

// In registers.  GPT: groups among a thread's V channels (W = V / GPT channels of each); NV: pixels of a thread at most.
// 400 x 256 x 256 bf16: 21.1 us, 5.0 TB/s of the 6.8 of a copy: a block's chain of loads, two sums and stores at 32
// warps an SM, about a third of its instructions the same for any number of pixels.
template <typename T, typename TY, int V, int GPT, int NV>
__global__ void __launch_bounds__(THREADS, V == 1 ? 3 : 4) held_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int W = V / GPT, NP = (V + 1) / 2;
    __shared__ Shared<GPT> sm;
    const Tile w = tile<V>(a);
    const T *x = static_cast<const T *>(a.x) + ((int64_t)w.b * a.P + w.p0 + w.row) * a.ldx + w.c;
    const int64_t step = (int64_t)w.rows * a.ldx;
    Vec<T, V> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i < w.n) v[i].load(x + i * step);

    float mean[GPT], rstd[GPT];
    {
        // pairs of channels: of one group, or (W = 1) of two
        Pair s[NP], q[NP];
#pragma unroll
        for (int k = 0; k < NP; ++k) s[k] = q[k] = pair(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < w.n) {
#pragma unroll
                for (int k = 0; k < NP; ++k) s[k] = add2(s[k], v[i].get2(k));
            }
        float own[GPT], m2[GPT];
        fold_pairs<V, GPT>(s, own);
        const float values = (float)(w.n * W), inv = w.n > 0 ? __fdividef(1.0f, values) : 0.0f;
#pragma unroll
        for (int g = 0; g < GPT; ++g) own[g] *= inv;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < w.n) {
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    const Pair d = add2(v[i].get2(k), pick_group<V, W>(own, k, -1.0f));
                    q[k] = fma2(d, d, q[k]);
                }
            }
        fold_pairs<V, GPT>(q, m2);
        merge<GPT>(a, w, sm, own, m2, values, mean, rstd);
    }
    if (w.n > 0) {
        Pair nm[NP], sc[NP], sh[NP];
        coefficients<V, GPT>(a, w.c, mean, rstd, nm, sc, sh);
        TY *y = static_cast<TY *>(a.y) + ((int64_t)w.b * a.P + w.p0 + w.row) * a.ldy + w.c;
        const int64_t ystep = (int64_t)w.rows * a.ldy;
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < w.n) apply_pixel<T, TY, V, act.value>(v[i], y + i * ystep, nm, sc, sh);
        });
    }
}

// In shared memory.  Each thread copies the vectors that it reads, so that only the sums need barriers.  128 x 784 x 128
// bf16: 13.2 us, 3.9 TB/s: all of x is read before anything is written.  1 x 64 x 512: 2.8 us, a chain of latencies.
template <typename T, typename TY, int V, int GPT>
__global__ void __launch_bounds__(THREADS, 3) shared_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int W = V / GPT, NP = V / 2, U = 4, BYTES = Vec<T, V>::BYTES;
    extern __shared__ __align__(16) uint8_t data[];
    __shared__ Shared<GPT> sm;
    const Tile w = tile<V>(a);
    const int64_t p = (int64_t)w.b * a.P + w.p0 + w.row;
    uint8_t *own_data = data + threadIdx.x * BYTES;
    {
        const T *x = static_cast<const T *>(a.x) + p * a.ldx + w.c;
        const int64_t step = (int64_t)w.rows * a.ldx;
#pragma unroll U
        for (int i = 0; i < w.n; ++i, x += step) copy_async<BYTES>(own_data + i * (THREADS * BYTES), x);
        asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
    }
    auto value = [&](int i) {
        Vec<T, V> v;
        v.load(reinterpret_cast<const T *>(own_data + i * (THREADS * BYTES)));
        return v;
    };
    float mean[GPT], rstd[GPT];
    {
        Pair s[NP], q[NP];
#pragma unroll
        for (int k = 0; k < NP; ++k) s[k] = q[k] = pair(0.0f, 0.0f);
#pragma unroll U
        for (int i = 0; i < w.n; ++i) {
            const Vec<T, V> v = value(i);
#pragma unroll
            for (int k = 0; k < NP; ++k) s[k] = add2(s[k], v.get2(k));
        }
        float own[GPT], m2[GPT];
        fold_pairs<V, GPT>(s, own);
        const float values = (float)(w.n * W), inv = w.n > 0 ? __fdividef(1.0f, values) : 0.0f;
#pragma unroll
        for (int g = 0; g < GPT; ++g) own[g] *= inv;
#pragma unroll U
        for (int i = 0; i < w.n; ++i) {
            const Vec<T, V> v = value(i);
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const Pair d = add2(v.get2(k), pick_group<V, W>(own, k, -1.0f));
                q[k] = fma2(d, d, q[k]);
            }
        }
        fold_pairs<V, GPT>(q, m2);
        merge<GPT>(a, w, sm, own, m2, values, mean, rstd);
    }
    if (w.n > 0) {
        Pair nm[NP], sc[NP], sh[NP];
        coefficients<V, GPT>(a, w.c, mean, rstd, nm, sc, sh);
        const int64_t ystep = (int64_t)w.rows * a.ldy;
        with_act(a.act, [&](auto act) {
            TY *y = static_cast<TY *>(a.y) + p * a.ldy + w.c;
#pragma unroll U
            for (int i = 0; i < w.n; ++i, y += ystep) apply_pixel<T, TY, V, act.value>(value(i), y, nm, sc, sh);
        });
    }
    if (a.chunks > 1) cluster_leave();
}

// In two readings, but for the pixels that the ring still holds at the second: where a slab is more than a block holds
// in registers (200 x 784 x 256 fp32: 60 us; 68 in the registers of clusters of four; 200 x 400 x 256: 30.1 and 35.5)
// and the slabs more than the SMs hold in shared memory.  256 x 1024 x 128, fp32 to bf16: 42.2 us, 4.8 TB/s.
template <typename T, typename TY, int V, int GPT>
__global__ void __launch_bounds__(THREADS, 4) reread_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int W = V / GPT, NP = (V + 1) / 2;
    extern __shared__ __align__(16) uint8_t data[];
    __shared__ Shared<GPT> sm;
    const Tile w = tile<V>(a);
    const int64_t p = (int64_t)w.b * a.P + w.p0 + w.row, step = (int64_t)w.rows * a.ldx;
    const T *x = static_cast<const T *>(a.x) + p * a.ldx + w.c;
    const Ring<T, V> ring(data);
    const int first = V > 1 ? ring.first(w.n) : w.n;        // what is still there at the second reading
    float mean[GPT], rstd[GPT];
    {
        Pair m[NP], q[NP];
        if constexpr (V == 1) channel_stats<T, V, 16>(x, step, w.n, m, q);
        else ring.stats(x, step, w.n, m, q);
        float own[GPT], m2[GPT];
        fold_channels<V, GPT>(m, q, w.n, own, m2);
        merge<GPT>(a, w, sm, own, m2, (float)w.n * (float)W, mean, rstd);
    }
    if (w.n > 0) {
        Pair nm[NP], sc[NP], sh[NP];
        coefficients<V, GPT>(a, w.c, mean, rstd, nm, sc, sh);
        with_act(a.act, [&](auto act) {
            apply_pixels<T, TY, V, V == 1 ? 8 : 4, act.value>(x, step, static_cast<TY *>(a.y) + p * a.ldy + w.c,
                                                              (int64_t)w.rows * a.ldy, first, w.n,
                                                              [&](int i) { return ring.read(i); }, nm, sc, sh);
        });
    }
    if (a.chunks > 1) cluster_leave();
}

// ---------------------------------------------------------------------------
// Two kernels, for images that no cluster could take alone: the statistics of
// every STREAM_CLUSTER chunks of an image, merged by a cluster; then each block
// merges its image's and applies them to its chunk.  2 x 252003 x 96 bf16 of 160:
// 63.7 us; the lines of its rows are 129 MB, read twice, a third of the second
// time from L2, and 97 MB are written: 4.9 TB/s of memory traffic.
// ---------------------------------------------------------------------------

template <typename T, int V, int GPT>
__global__ void __launch_bounds__(THREADS, 4) chunk_stats_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int W = V / GPT, NP = (V + 1) / 2;
    __shared__ __align__(16) uint8_t data[V == 1 ? 16 : Ring<T, V>::SIZE];
    __shared__ Shared<GPT> sm;
    const Tile w = tile<V>(a);
    float own[GPT], m2[GPT], mean[GPT];
    {
        Pair m[NP], q[NP];
        const T *x = static_cast<const T *>(a.x) + ((int64_t)w.b * a.P + w.p0 + w.row) * a.ldx + w.c;
        if constexpr (V == 1) channel_stats<T, V, 16>(x, (int64_t)w.rows * a.ldx, w.n, m, q);
        else Ring<T, V>(data).stats(x, (int64_t)w.rows * a.ldx, w.n, m, q);
        fold_channels<V, GPT>(m, q, w.n, own, m2);
    }
    merge_block<GPT>(a, w, sm, own, (float)w.n * (float)W, mean, m2);
    const int first = w.rank / STREAM_CLUSTER * STREAM_CLUSTER;
    merge_cluster<GPT>(a, w, sm, first, STREAM_CLUSTER, mean, m2);
    if (w.rank == first) {
        float2 *part = a.part + ((int64_t)w.b * (a.chunks / STREAM_CLUSTER) + w.rank / STREAM_CLUSTER) * a.G;
        for (int g = threadIdx.x; g < a.groups; g += THREADS) part[w.slab * a.groups + g] = sm.all[g];
    }
    cluster_leave();
}

template <typename T, typename TY, int V, int GPT>
__global__ void __launch_bounds__(THREADS, 4) chunk_apply_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int NP = (V + 1) / 2, EACH = (STREAM_BLOCKS / STREAM_CLUSTER + 31) / 32;
    __shared__ float2 all[MAX_SLAB_GROUPS];
    const Tile w = tile<V>(a);
    const int parts = a.chunks / STREAM_CLUSTER, lane = threadIdx.x & 31;
    const float2 *part = a.part + (int64_t)w.b * parts * a.G + w.slab * a.groups;
    for (int g = threadIdx.x >> 5; g < a.groups; g += THREADS / 32) {           // a warp per group
        float2 t[EACH];
        float n[EACH], s = 0.0f, q = 0.0f;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int k = lane + 32 * e;
            t[e] = k < parts ? part[(int64_t)k * a.G + g] : make_float2(0.0f, 0.0f);
            n[e] = k < parts ? (float)(min(a.P, (k + 1) * STREAM_CLUSTER * a.ppc) - min(a.P, k * STREAM_CLUSTER * a.ppc)) * (float)a.Cg
                             : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e) s = fmaf(n[e], t[e].x, s);
        const float mean = warp_sum(s) * a.inv_total;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const float d = t[e].x - mean;
            if (n[e] > 0.0f) q += fmaf(d * d, n[e], t[e].y);
        }
        const float rstd = rsqrtf(fmaf(warp_sum(q), a.inv_total, a.eps));
        if (lane == 0) {
            all[g] = make_float2(mean, rstd);
            const int64_t at = (int64_t)w.b * a.G + w.slab * a.groups + g;
            if (w.rank == 0 && a.mean) a.mean[at] = mean;
            if (w.rank == 0 && a.rstd) a.rstd[at] = rstd;
        }
    }
    __syncthreads();
    if (w.n == 0) return;
    Pair nm[NP], sc[NP], sh[NP];
    {
        float mean[GPT], rstd[GPT];
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            const float2 t = all[a.by_per.div(w.lane * GPT + g)];
            mean[g] = t.x;
            rstd[g] = t.y;
        }
        coefficients<V, GPT>(a, w.c, mean, rstd, nm, sc, sh);
    }
    const int64_t p = (int64_t)w.b * a.P + w.p0 + w.row;
    with_act(a.act, [&](auto act) {
        apply_pixels<T, TY, V, V == 1 ? 8 : 4, act.value>(static_cast<const T *>(a.x) + p * a.ldx + w.c,
                                                          (int64_t)w.rows * a.ldx, static_cast<TY *>(a.y) + p * a.ldy + w.c,
                                                          (int64_t)w.rows * a.ldy, w.n, w.n, [](int) { return Vec<T, V>(); }, nm, sc, sh);
    });
}

// The kernels of a plan: one, or the two of images in chunks.
struct Kernels {
    void (*one)(Args), (*stats)(Args), (*apply)(Args);
};
template <typename T, typename TY, int V, int GPT>
static Kernels kernels_of(Way way) {
    Kernels k = {way == HELD ? held_kernel<T, TY, V, GPT, V == 1 ? 32 : 8> : reread_kernel<T, TY, V, GPT>,
                 chunk_stats_kernel<T, V, GPT>, chunk_apply_kernel<T, TY, V, GPT>};
    if constexpr (V > 1)
        if (way == SHARED) k.one = shared_kernel<T, TY, V, GPT>;
    return k;
}

template <typename T, typename TY>
static minw_status forward(Args a, int V, cudaStream_t s) {
    Plan pl;
    if (plan(a, pl, (int)sizeof(T), 0, V)) {
        Kernels k = pl.V == 1    ? kernels_of<T, TY, 1, 1>(pl.way)
                    : pl.GPT == 1 ? kernels_of<T, TY, 4, 1>(pl.way)
                    : pl.GPT == 2 ? kernels_of<T, TY, 4, 2>(pl.way)
                                  : kernels_of<T, TY, 4, 4>(pl.way);
        if constexpr (sizeof(T) == 2 && sizeof(TY) == 2)
            if (pl.V == 8)
                k = pl.GPT == 1   ? kernels_of<T, TY, 8, 1>(pl.way)
                    : pl.GPT == 2 ? kernels_of<T, TY, 8, 2>(pl.way)
                                  : kernels_of<T, TY, 8, 4>(pl.way);
        if (pl.way != CHUNKS) {
            const int64_t blocks = (int64_t)a.B * a.slabs * a.chunks;
            if (blocks >= (1ll << 31)) return MINW_EUNSUPPORTED;
            return launch_cluster(k.one, blocks, a.chunks, pl.smem, s, a) == cudaSuccess ? launch_status() : launch_failed();
        }
        int64_t blocks;
        if (!in_chunks(a, true, blocks)) return MINW_EUNSUPPORTED;
        if (launch_cluster(k.stats, blocks, STREAM_CLUSTER, 0, s, a) != cudaSuccess || launch(k.apply, blocks, s, a) != cudaSuccess)
            return launch_failed();
        return launch_status();
    }
    lanes(a, V);
    void (*stat)(Args) = V == 4 ? stat_kernel<T, 4> : stat_kernel<T, 1>;
    void (*apply)(Args) = V == 4 ? apply_kernel<T, TY, 4> : apply_kernel<T, TY, 1>;
    if constexpr (sizeof(T) == 2 && sizeof(TY) == 2)
        if (V == 8) {
            stat = stat_kernel<T, 8>;
            apply = apply_kernel<T, TY, 8>;
        }
    int64_t blocks;
    if (!in_chunks(a, false, blocks)) return MINW_EUNSUPPORTED;
    if (launch(stat, blocks, s, a) != cudaSuccess || launch(stat_merge_kernel, (int64_t)a.B * a.G, s, a) != cudaSuccess ||
        launch(apply, blocks, s, a) != cudaSuccess)
        return launch_failed();
    return launch_status();
}

}  // namespace gn
}  // namespace minw

using namespace minw;
using namespace minw_host;

extern "C" {

size_t minw_group_norm_workspace_bytes(int32_t B, int64_t P, int32_t C, int32_t G, int32_t backward) {
    if (B <= 0 || P <= 0 || C <= 0 || G <= 0 || C % G != 0 || P >= (1ll << 30)) return 0;
    return gn::layout(B, P, C, G, backward != 0).total;
}

minw_status minw_group_norm(const void *x, int32_t x_type, int64_t ldx, const float *gamma, const float *beta,
                            int32_t B, int64_t P, int32_t C, int32_t G, float eps, int32_t act, void *y,
                            int32_t y_type, int64_t ldy, float *mean, float *rstd, void *workspace,
                            size_t workspace_bytes, void *stream) {
    if ((B != 0 && (!x || !y)) || B < 0 || P < 1 || C < 1 || G < 1 || C % G != 0 || ldx < C || ldy < C) return MINW_EINVAL;
    if (!gn::valid_type(x_type) || !gn::valid_type(y_type) || act < MINW_ACT_NONE || act > MINW_ACT_SILU)
        return MINW_EINVAL;
    if (!(eps >= 0.0f && isfinite(eps))) return MINW_EINVAL;
    if (!gn::fits(x, 1, x_type, 1) || !gn::fits(y, 1, y_type, 1) || !gn::in_place_ok(x, x_type, ldx, y, y_type, ldy))
        return MINW_EINVAL;
    if (!on_floats(gamma, beta, mean, rstd)) return MINW_EINVAL;
    if (P >= (1ll << 30)) return MINW_EUNSUPPORTED;
    if (B == 0) return MINW_OK;
    const gn::Layout l = gn::layout(B, P, C, G, false);
    if (!workspace || !aligned16(workspace) || workspace_bytes < l.total) return MINW_EINVAL;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    gn::Args a{};
    a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy; a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd;
    a.wide_affine = gamma && beta && aligned16(gamma) && aligned16(beta);
    a.B = B; a.P = (int)P; a.C = C; a.G = G; a.Cg = C / G; a.act = act; a.eps = eps;
    a.part = reinterpret_cast<float2 *>(ws + l.part);
    a.stat = reinterpret_cast<float2 *>(ws + l.stat);
    int V = x_type == MINW_BF16 && y_type == MINW_BF16 ? 8 : 4;       // 16 bytes of the wider type
    while (V > 1 && (C % V != 0 || !gn::fits(x, ldx, x_type, V) || !gn::fits(y, ldy, y_type, V))) V = V == 8 ? 4 : 1;
    cudaStream_t s = (cudaStream_t)stream;
    if (x_type == MINW_BF16)
        return y_type == MINW_BF16 ? gn::forward<uint16_t, uint16_t>(a, V, s) : gn::forward<uint16_t, float>(a, V, s);
    return y_type == MINW_BF16 ? gn::forward<float, uint16_t>(a, V, s) : gn::forward<float, float>(a, V, s);
}

}  // extern "C"
