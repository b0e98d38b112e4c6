// group_norm_bwd.cu -- backward of the group norm with an activation on
// channels-last rows (group_norm.cuh: tiles and plans).  The two sums over a
// group follow from the channel sums that dgamma and dbeta need anyway.
#include "group_norm.cuh"

namespace minw {
namespace gn {

// ---------------------------------------------------------------------------
// Streaming backward: the channel sums per chunk, merged per image, then a
// second pass over x and dy.  2 x 251001 x 64 bf16, SiLU: 62.4 us, 5.1 TB/s of the
// 320 MB that two readings and a writing move.
// ---------------------------------------------------------------------------

// What a thread's V channels need, in pairs: minus the means, scale = rstd gamma, beta.  With t = x - mean, z = scale t +
// beta; the sums are those of dz and dz t (times rstd at their end, dgamma), and dx = scale dz - rstd s1 - t rstd^2 s2.
template <int V>
struct Coef {
    static constexpr int NP = (V + 1) / 2;
    Pair nm[NP], sc[NP], be[NP];

    // in two steps, so that the pixels' loads can be on their way between
    float g[V], h[V], mean[V], rstd[V];
    __device__ __forceinline__ void fetch(const Args &a, int b, int c) {
        load_affine<V>(a, c, g, h);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int64_t at = (int64_t)b * a.G + a.by_Cg.div(c + i);
            mean[i] = a.mean_in[at];
            rstd[i] = a.rstd_in[at];
        }
    }
    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = -mean[i];
            g[i] *= rstd[i];
        }
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            nm[k] = pick<V>(mean, k);
            sc[k] = pick<V>(g, k);
            be[k] = pick<V>(h, k);
        }
    }
    __device__ __forceinline__ void load(const Args &a, int b, int c) {
        fetch(a, b, c);
        finish();
    }
};

// Sums of dz and dz t of one pixel's channels.
template <int ACT, int V, typename X, typename D>
__device__ __forceinline__ void add_pixel(const X &x, const D &dy, const Coef<V> &co, Pair *db, Pair *dg) {
#pragma unroll
    for (int k = 0; k < Coef<V>::NP; ++k) {
        const Pair t = add2(x.get2(k), co.nm[k]);
        const Pair dz = act_grad2<ACT>(fma2(t, co.sc[k], co.be[k]), dy.get2(k));
        db[k] = add2(db[k], dz);
        dg[k] = fma2(dz, t, dg[k]);
    }
}

// dx of one pixel: n1 = - rstd s1 and n2 = - rstd^2 s2 of its channels' groups in pairs.
template <int ACT, int V, typename X, typename D>
__device__ __forceinline__ X pixel_gradient(const X &x, const D &dy, const Coef<V> &co, const Pair *n1, const Pair *n2) {
    float o[2 * Coef<V>::NP];
#pragma unroll
    for (int k = 0; k < Coef<V>::NP; ++k) {
        const Pair t = add2(x.get2(k), co.nm[k]);
        const Pair dz = act_grad2<ACT>(fma2(t, co.sc[k], co.be[k]), dy.get2(k));
        const float2 h = halves(fma2(co.sc[k], dz, fma2(t, n2[k], n1[k])));
        o[2 * k] = h.x;
        o[2 * k + 1] = h.y;
    }
    X r;
    r.set(o);
    return r;
}

// Sums over a thread's n pixels, `step` values apart; co has been fetched.
template <typename T, typename TD, int V, int U>
__device__ __forceinline__ void channel_sums(int act, const T *x, int64_t xstep, const TD *dy, int64_t dstep, int n,
                                             Coef<V> &co, Pair *db, Pair *dg) {
#pragma unroll
    for (int k = 0; k < Coef<V>::NP; ++k) db[k] = dg[k] = pair(0.0f, 0.0f);
    with_act(act, [&](auto act_) {
        const T *px = x;
        const TD *pd = dy;
        Vec<T, V> v[U];
        Vec<TD, V> d[U];
        batches<U>(
            n,
            [&](int u) {
                v[u].load(px);
                d[u].load(pd);
                px += xstep;
                pd += dstep;
            },
            [&] { co.finish(); }, [&](int u) { add_pixel<act_.value, V>(v[u], d[u], co, db, dg); });
    });
}

// The same through a ring of asynchronous copies: eight pixels of a thread in flight, and the last ones of it, from
// first() on, stay there.  Each thread reads its own copies.
template <typename T, typename TD, int V>
struct RingBwd {
    static constexpr int U = 4, XB = Vec<T, V>::BYTES, DB = Vec<TD, V>::BYTES;
    uint8_t *x, *dy;
    __device__ __forceinline__ explicit RingBwd(uint8_t *shared)
        : x(shared + threadIdx.x * XB), dy(shared + RING_PIXELS * THREADS * XB + threadIdx.x * DB) {}
    static __device__ __forceinline__ int at(int i) { return (i & (RING_PIXELS - 1)) * THREADS; }
    static __device__ __forceinline__ int first(int n) { return max((n + U - 1) / U * U - RING_PIXELS, 0); }
    __device__ __forceinline__ void read(int i, Vec<T, V> &v, Vec<TD, V> &d) const {
        v.load(reinterpret_cast<const T *>(x + at(i) * XB));
        d.load(reinterpret_cast<const TD *>(dy + at(i) * DB));
    }
    __device__ __forceinline__ void sums(int act, const T *px, int64_t xstep, const TD *pd, int64_t dstep, int n, Coef<V> &co,
                                         Pair *db, Pair *dg) const {
        auto fetch = [&](int i0) {                              // pixels i0 .. i0 + U - 1, those that there are
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u < n) {
                    copy_async<XB>(x + at(i0 + u) * XB, px + u * xstep);
                    copy_async<DB>(dy + at(i0 + u) * DB, pd + u * dstep);
                }
            px += U * xstep;
            pd += U * dstep;
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        static_assert(RING_PIXELS == 2 * U, "two fetches in flight");
        fetch(0);
        fetch(U);
#pragma unroll
        for (int k = 0; k < Coef<V>::NP; ++k) db[k] = dg[k] = pair(0.0f, 0.0f);
        co.finish();
        with_act(act, [&](auto act_) {
            for (int i0 = 0; i0 < n; i0 += U) {
                asm volatile("cp.async.wait_group 1;" ::: "memory");
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i0 + u < n) {
                        Vec<T, V> v;
                        Vec<TD, V> d;
                        read(i0 + u, v, d);
                        add_pixel<act_.value, V>(v, d, co, db, dg);
                    }
                fetch(i0 + RING_PIXELS);
            }
        });
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
};

// dx of a thread's n pixels, those from `first` on from kept(i, x, dy).
template <typename T, typename TD, int V, int U, typename K>
__device__ __forceinline__ void gradient_pixels(int act, const T *x, int64_t xstep, const TD *dy, int64_t dstep, T *dx,
                                                int64_t ostep, int first, int n, K kept, const Coef<V> &co, const Pair *n1,
                                                const Pair *n2) {
    with_act(act, [&](auto act_) {
        const T *px = x;
        const TD *pd = dy;
        T *po = dx;
        Vec<T, V> v[U];
        Vec<TD, V> d[U];
        batches<U>(
            first,
            [&](int u) {
                v[u].load(px);
                d[u].load(pd);
                px += xstep;
                pd += dstep;
            },
            [&] {
#pragma unroll 4
                for (int i = first; i < n; ++i) {
                    Vec<T, V> kv;
                    Vec<TD, V> kd;
                    kept(i, kv, kd);
                    pixel_gradient<act_.value, V>(kv, kd, co, n1, n2).store(dx + i * ostep);
                }
            },
            [&](int u) {
                pixel_gradient<act_.value, V>(v[u], d[u], co, n1, n2).store(po);
                po += ostep;
            });
    });
}

// A thread's channel sums into its row of the block's.
template <int V>
__device__ __forceinline__ void put_sums(float2 *at, const Pair *db, const Pair *dg) {
#pragma unroll
    for (int k = 0; k < (V + 1) / 2; ++k) {
        const float2 b = halves(db[k]), g = halves(dg[k]);
        at[2 * k] = make_float2(b.x, g.x);
        if (V > 1) at[2 * k + 1] = make_float2(b.y, g.y);
    }
}

template <typename T, typename TD, int V>
__global__ void __launch_bounds__(THREADS, 2) bwd_sum_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    extern __shared__ __align__(16) uint8_t data[];
    __shared__ float2 red[THREADS * V];
    const Place w = place<V>(a, blockIdx.x);
    const int W = a.L * V;
    if (w.row < w.rows) {
        Pair db[Coef<V>::NP], dg[Coef<V>::NP];
        Coef<V> co;
        if (w.n > 0) co.fetch(a, w.b, w.c);
        const int64_t p = (int64_t)w.b * a.P + w.p0 + w.row;
        const T *x = static_cast<const T *>(a.x) + p * a.ldx + w.c;
        const TD *dy = static_cast<const TD *>(a.dy) + p * a.lddy + w.c;
        if constexpr (V == 1) channel_sums<T, TD, V, 8>(a.act, x, w.rows * a.ldx, dy, w.rows * a.lddy, w.n, co, db, dg);
        else RingBwd<T, TD, V>(data).sums(a.act, x, w.rows * a.ldx, dy, w.rows * a.lddy, w.n, co, db, dg);
        put_sums<V>(red + w.row * W + w.lane * V, db, dg);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < W; e += THREADS) {
        const int c = w.slab * W + e;
        if (c >= a.C) break;
        float s0 = 0.0f, s1 = 0.0f;
        for (int r = 0; r < w.rows; ++r) {
            s0 += red[r * W + e].x;
            s1 += red[r * W + e].y;
        }
        a.part[((int64_t)w.b * a.chunks + w.chunk) * a.C + c] =
            make_float2(s0, s1 * a.rstd_in[(int64_t)w.b * a.G + c / a.Cg]);
    }
}

// Block = one image's group: its channels' sums over the chunks, then s1 and s2.
__global__ void __launch_bounds__(THREADS) bwd_merge_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    __shared__ float2 red[THREADS / 32];
    const int b = (int)(blockIdx.x / a.G), g = (int)(blockIdx.x % a.G), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float s1 = 0.0f, s2 = 0.0f;
    for (int e = warp; e < a.Cg; e += THREADS / 32) {          // a warp per channel
        const int c = g * a.Cg + e;
        float db = 0.0f, dg = 0.0f;
        for (int k = lane; k < a.chunks; k += 32) {
            const float2 t = a.part[((int64_t)b * a.chunks + k) * a.C + c];
            db += t.x;
            dg += t.y;
        }
        db = warp_sum(db);
        dg = warp_sum(dg);
        if (lane == 0) a.chan[(int64_t)b * a.C + c] = make_float2(db, dg);
        const float ga = a.gamma ? a.gamma[c] : 1.0f;
        s1 = fmaf(ga, db, s1);
        s2 = fmaf(ga, dg, s2);
    }
    if (lane == 0) red[warp] = make_float2(s1, s2);
    __syncthreads();
    if (threadIdx.x == 0) {
        s1 = s2 = 0.0f;
        for (int k = 0; k < THREADS / 32; ++k) {
            s1 += red[k].x;
            s2 += red[k].y;
        }
        const float n = (float)a.P * (float)a.Cg;
        a.stat[blockIdx.x] = make_float2(s1 / n, s2 / n);
    }
}

template <typename T, typename TD, int V>
__global__ void __launch_bounds__(THREADS, 2) bwd_apply_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    const Place w = place<V>(a, (int64_t)gridDim.x - 1 - blockIdx.x);
    if (w.n == 0) return;
    Coef<V> co;
    co.load(a, w.b, w.c);
    Pair n1[Coef<V>::NP], n2[Coef<V>::NP];
    {
        float s1[V], s2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int64_t at = (int64_t)w.b * a.G + (w.c + i) / a.Cg;
            const float2 t = a.stat[at];
            const float r = a.rstd_in[at];
            s1[i] = -t.x * r;
            s2[i] = -t.y * r * r;
        }
#pragma unroll
        for (int k = 0; k < Coef<V>::NP; ++k) {
            n1[k] = pick<V>(s1, k);
            n2[k] = pick<V>(s2, k);
        }
    }
    // from the last pixel to the first: what the sums read last is what L2 still holds (2 x 251001 x 64: 64.8 us for 67.1)
    const int64_t p = (int64_t)w.b * a.P + w.p0 + w.row + (int64_t)(w.n - 1) * w.rows;
    gradient_pixels<T, TD, V, V == 1 ? 8 : 4>(a.act, static_cast<const T *>(a.x) + p * a.ldx + w.c, -w.rows * a.ldx,
                                              static_cast<const TD *>(a.dy) + p * a.lddy + w.c, -w.rows * a.lddy,
                                              static_cast<T *>(a.y) + p * a.ldy + w.c, -w.rows * a.ldy, w.n, w.n, [](int, auto &, auto &) {}, co, n1, n2);
}

// ---------------------------------------------------------------------------
// One kernel.
// ---------------------------------------------------------------------------

template <int V>
struct Shared {
    float2 red[THREADS * V];               // rows x channels, then segments x channels
    float2 group[MAX_SLAB_GROUPS];
    float2 scaled[THREADS];                // totals times gamma, where a thread has no more than one channel
    float rstd[MAX_SLAB_GROUPS];           // of the slab's groups

    __device__ __forceinline__ void load_rstd(const Args &a, const Tile &w) {
        for (int g = threadIdx.x; g < a.groups; g += THREADS) rstd[g] = a.rstd_in[(int64_t)w.b * a.G + w.slab * a.groups + g];
    }
};
static_assert(sizeof(Shared<8>) == 8 * THREADS * 9 + 12 * MAX_SLAB_GROUPS, "plan() counts on it");

// n1 and n2 of a thread's channels from its sums: the block's rows, the cluster's blocks, the groups' channels, all
// in a fixed order; and the image's channel sums for dgamma and dbeta.  Afterwards a cluster has arrived at its end.
template <int V>
__device__ __forceinline__ void totals(const Args &a, const Tile &w, Shared<V> &sm, const Pair *db, const Pair *dg, Pair *n1,
                                       Pair *n2) {
    const int CW = a.L * V;                                // channels of the slab
    float2 *red = sm.red;
    const bool few = CW <= THREADS;
    const float gamma = few && a.gamma && (int)threadIdx.x < CW ? a.gamma[w.slab * CW + threadIdx.x] : 1.0f;      // early
    if (w.row < w.rows) put_sums<V>(red + w.row * CW + w.lane * V, db, dg);
    __syncthreads();
    // `seg` threads a channel, each every so many rows (into the row of its number)
    for (int s = a.by_channels.div((int)threadIdx.x), c = (int)threadIdx.x - s * CW; s < a.seg;) {
        float2 t = red[s * CW + c];
        for (int r = s + a.seg; r < w.rows; r += a.seg) {
            t.x += red[r * CW + c].x;
            t.y += red[r * CW + c].y;
        }
        red[s * CW + c] = t;
        c += THREADS;                                      // more channels than threads: one segment
        if (a.seg > 1 || c >= CW) break;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < CW; c += THREADS) {
        float2 t = red[c];
        for (int s = 1; s < a.seg; ++s) {
            t.x += red[s * CW + c].x;
            t.y += red[s * CW + c].y;
        }
        t.y *= sm.rstd[a.by_Cg.div(c)];
        red[c] = t;
        if (few) sm.scaled[c] = make_float2(gamma * t.x, gamma * t.y);
    }
    float2 *tot = red;
    if (a.chunks > 1) {
        // the cluster's blocks: their sums stay in place while the totals go behind them
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        tot = red + CW;
        for (int c = threadIdx.x; c < CW; c += THREADS) {
            float2 u[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                u[k] = k < a.chunks ? *cluster.map_shared_rank(&red[c], k) : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int k = 1; k < 8; ++k) {
                u[0].x += u[k].x;
                u[0].y += u[k].y;
            }
            tot[c] = u[0];
            if (few) sm.scaled[c] = make_float2(gamma * u[0].x, gamma * u[0].y);
        }
        cluster_done_reading();
    }
    __syncthreads();
    if (w.rank == 0)
        for (int c = threadIdx.x; c < CW; c += THREADS) a.chan[(int64_t)w.b * a.C + w.slab * CW + c] = tot[c];
    for (int g = threadIdx.x >> 5; g < a.groups; g += THREADS / 32) {
        float s1 = 0.0f, s2 = 0.0f;
        for (int k = threadIdx.x & 31; k < a.Cg; k += 32) {
            float2 t = sm.scaled[few ? g * a.Cg + k : 0];
            if (!few) {
                const float gk = a.gamma ? a.gamma[w.slab * CW + g * a.Cg + k] : 1.0f;
                t = make_float2(gk * tot[g * a.Cg + k].x, gk * tot[g * a.Cg + k].y);
            }
            s1 += t.x;
            s2 += t.y;
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if ((threadIdx.x & 31) == 0) {
            const float r = -sm.rstd[g] * a.inv_total;
            sm.group[g] = make_float2(s1 * r, s2 * r * sm.rstd[g]);
        }
    }
    __syncthreads();
    float f1[V], f2[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 t = sm.group[a.by_Cg.div(w.lane * V + i)];
        f1[i] = t.x;
        f2[i] = t.y;
    }
#pragma unroll
    for (int k = 0; k < (V + 1) / 2; ++k) {
        n1[k] = pick<V>(f1, k);
        n2[k] = pick<V>(f2, k);
    }
}

// In registers: at most NV pixels of each thread.  256 x 256 x 256 bf16: 30.4 us, 3.3 TB/s: 16 warps an SM, and each has
// its loads, sums and stores one after the other.
template <typename T, typename TD, int V, int NV>
__global__ void __launch_bounds__(THREADS, 2) held_bwd_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int NP = Coef<V>::NP;
    __shared__ Shared<V> sm;
    const Tile w = tile<V>(a);
    const int64_t p = (int64_t)w.b * a.P + w.p0 + w.row, xstep = (int64_t)w.rows * a.ldx, dstep = (int64_t)w.rows * a.lddy;
    const T *x = static_cast<const T *>(a.x) + p * a.ldx + w.c;
    const TD *dy = static_cast<const TD *>(a.dy) + p * a.lddy + w.c;
    Vec<T, V> v[NV];
    Vec<TD, V> d[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i < w.n) {
            v[i].load(x + i * xstep);
            d[i].load(dy + i * dstep);
        }
    Coef<V> co;
    co.load(a, w.b, w.c);
    sm.load_rstd(a, w);
    Pair n1[NP], n2[NP];
    {
        Pair db[NP], dg[NP];
#pragma unroll
        for (int k = 0; k < NP; ++k) db[k] = dg[k] = pair(0.0f, 0.0f);
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < w.n) add_pixel<act.value, V>(v[i], d[i], co, db, dg);
        });
        totals<V>(a, w, sm, db, dg, n1, n2);
    }
    T *dx = static_cast<T *>(a.y) + p * a.ldy + w.c;
    const int64_t ostep = (int64_t)w.rows * a.ldy;
    with_act(a.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < w.n) pixel_gradient<act.value, V>(v[i], d[i], co, n1, n2).store(dx + i * ostep);
    });
}

// In shared memory.  Each thread copies the vectors that it reads, so that only the sums need barriers.
template <typename T, typename TD, int V>
__global__ void __launch_bounds__(THREADS, 2) shared_bwd_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int NP = V / 2, U = 2, BYTES = Vec<T, V>::BYTES + Vec<TD, V>::BYTES, XB = Vec<T, V>::BYTES;
    extern __shared__ __align__(16) uint8_t data[];
    __shared__ Shared<V> sm;
    const Tile w = tile<V>(a);
    const int64_t p = (int64_t)w.b * a.P + w.p0 + w.row;
    // a pixel's vectors of all threads: x, then dy
    uint8_t *own_x = data + threadIdx.x * XB, *own_d = data + THREADS * XB + threadIdx.x * (BYTES - XB);
    {
        const T *x = static_cast<const T *>(a.x) + p * a.ldx + w.c;
        const TD *dy = static_cast<const TD *>(a.dy) + p * a.lddy + w.c;
        const int64_t xstep = (int64_t)w.rows * a.ldx, dstep = (int64_t)w.rows * a.lddy;
#pragma unroll 4
        for (int i = 0; i < w.n; ++i, x += xstep, dy += dstep) {
            copy_async<XB>(own_x + i * (THREADS * BYTES), x);
            copy_async<BYTES - XB>(own_d + i * (THREADS * BYTES), dy);
        }
    }
    Coef<V> co;
    co.load(a, w.b, w.c);
    sm.load_rstd(a, w);
    asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
    auto pixel = [&](int i, Vec<T, V> &v, Vec<TD, V> &d) {
        v.load(reinterpret_cast<const T *>(own_x + i * (THREADS * BYTES)));
        d.load(reinterpret_cast<const TD *>(own_d + i * (THREADS * BYTES)));
    };
    Pair n1[NP], n2[NP];
    {
        Pair db[NP], dg[NP];
#pragma unroll
        for (int k = 0; k < NP; ++k) db[k] = dg[k] = pair(0.0f, 0.0f);
        with_act(a.act, [&](auto act) {
#pragma unroll U
            for (int i = 0; i < w.n; ++i) {
                Vec<T, V> v;
                Vec<TD, V> d;
                pixel(i, v, d);
                add_pixel<act.value, V>(v, d, co, db, dg);
            }
        });
        totals<V>(a, w, sm, db, dg, n1, n2);
    }
    const int64_t ostep = (int64_t)w.rows * a.ldy;
    with_act(a.act, [&](auto act) {
        T *dx = static_cast<T *>(a.y) + p * a.ldy + w.c;
#pragma unroll U
        for (int i = 0; i < w.n; ++i, dx += ostep) {
            Vec<T, V> v;
            Vec<TD, V> d;
            pixel(i, v, d);
            pixel_gradient<act.value, V>(v, d, co, n1, n2).store(dx);
        }
    });
    if (a.chunks > 1) cluster_leave();
}

// In two readings, but for the pixels that the ring still holds at the second (128 x 3136 x 64, SiLU: 50.9 us; 53.5 with
// both readings into registers).  Bound by latency and by SiLU's approximate instructions, four for a value: 22 us.
template <typename T, typename TD, int V>
__global__ void __launch_bounds__(THREADS, 2) reread_bwd_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int NP = Coef<V>::NP, U = V == 8 ? 4 : 8;
    extern __shared__ __align__(16) uint8_t data[];
    __shared__ Shared<V> sm;
    const Tile w = tile<V>(a);
    const int64_t p = (int64_t)w.b * a.P + w.p0 + w.row, xstep = (int64_t)w.rows * a.ldx, dstep = (int64_t)w.rows * a.lddy;
    const T *x = static_cast<const T *>(a.x) + p * a.ldx + w.c;
    const TD *dy = static_cast<const TD *>(a.dy) + p * a.lddy + w.c;
    Coef<V> co;
    co.fetch(a, w.b, w.c);
    Pair n1[NP], n2[NP];
    const RingBwd<T, TD, V> ring(data);
    const int first = V == 1 ? w.n : ring.first(w.n);
    {
        Pair db[NP], dg[NP];
        if constexpr (V == 1) channel_sums<T, TD, V, 8>(a.act, x, xstep, dy, dstep, w.n, co, db, dg);
        else ring.sums(a.act, x, xstep, dy, dstep, w.n, co, db, dg);
        sm.load_rstd(a, w);
        totals<V>(a, w, sm, db, dg, n1, n2);
    }
    gradient_pixels<T, TD, V, U>(a.act, x, xstep, dy, dstep, static_cast<T *>(a.y) + p * a.ldy + w.c,
                                 (int64_t)w.rows * a.ldy, first, w.n,
                                 [&](int i, Vec<T, V> &v, Vec<TD, V> &d) { ring.read(i, v, d); }, co, n1, n2);
    if (a.chunks > 1) cluster_leave();
}

// dbeta, dgamma: the images' channel sums.  Eight channels (64 bytes) of a block, 32 images side by side, eight loads of a
// thread at a time: a chain of latencies (the backward of 256 x 256 x 256 bf16: 30.4 us; 31.9 with 8 images side by side
// and 32 loads of a thread).
constexpr int AFFINE_CHANNELS = 8;
__global__ void __launch_bounds__(THREADS) affine_grad_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int ROWS = THREADS / AFFINE_CHANNELS, U = 8;
    __shared__ float2 red[THREADS / 32][AFFINE_CHANNELS];
    const int own = threadIdx.x % AFFINE_CHANNELS, c = (int)blockIdx.x * AFFINE_CHANNELS + own;
    float db = 0.0f, dg = 0.0f;
    for (int64_t b = threadIdx.x / AFFINE_CHANNELS; b < a.B; b += U * ROWS) {
        float2 t[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            t[u] = c < a.C && b + u * ROWS < a.B ? a.chan[(b + u * ROWS) * a.C + c] : make_float2(0.0f, 0.0f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            db += t[u].x;
            dg += t[u].y;
        }
    }
#pragma unroll
    for (int d = AFFINE_CHANNELS; d < 32; d *= 2) {
        db += __shfl_xor_sync(0xffffffffu, db, d);
        dg += __shfl_xor_sync(0xffffffffu, dg, d);
    }
    if ((threadIdx.x & 31) < AFFINE_CHANNELS) red[threadIdx.x >> 5][own] = make_float2(db, dg);
    __syncthreads();
    if (threadIdx.x < AFFINE_CHANNELS && c < a.C) {
        db = dg = 0.0f;
#pragma unroll
        for (int k = 0; k < THREADS / 32; ++k) {
            db += red[k][own].x;
            dg += red[k][own].y;
        }
        if (a.dbeta) a.dbeta[c] = db;
        if (a.dgamma) a.dgamma[c] = dg;
    }
}

template <typename T, typename TD, int V>
static void (*kernel_of(Way way))(Args) {
    if constexpr (V > 1)
        if (way == SHARED) return shared_bwd_kernel<T, TD, V>;
    return way == HELD ? held_bwd_kernel<T, TD, V, V == 1 ? 32 : 8> : reread_bwd_kernel<T, TD, V>;
}

template <typename T, typename TD>
static minw_status backward(Args a, int V, cudaStream_t s) {
    Plan pl;
    if (Args f = a; plan(f, pl, (int)sizeof(T), (int)sizeof(TD), V)) {
        const int64_t blocks = (int64_t)f.B * f.slabs * f.chunks;
        if (blocks >= (1ll << 31)) return MINW_EUNSUPPORTED;
        void (*kern)(Args) = pl.V == 1 ? kernel_of<T, TD, 1>(pl.way) : kernel_of<T, TD, 4>(pl.way);
        if constexpr (sizeof(T) == 2 && sizeof(TD) == 2)
            if (pl.V == 8) kern = kernel_of<T, TD, 8>(pl.way);
        if (launch_cluster(kern, blocks, f.chunks, pl.smem, s, f) != cudaSuccess) return launch_failed();
    } else {
        lanes(a, V);
        void (*sum)(Args) = V == 4 ? bwd_sum_kernel<T, TD, 4> : bwd_sum_kernel<T, TD, 1>;
        void (*apply)(Args) = V == 4 ? bwd_apply_kernel<T, TD, 4> : bwd_apply_kernel<T, TD, 1>;
        if constexpr (sizeof(T) == 2 && sizeof(TD) == 2)
            if (V == 8) {
                sum = bwd_sum_kernel<T, TD, 8>;
                apply = bwd_apply_kernel<T, TD, 8>;
            }
        int64_t blocks;
        if (!in_chunks(a, false, blocks)) return MINW_EUNSUPPORTED;
        const int ring = V > 1 ? RING_PIXELS * THREADS * V * (int)(sizeof(T) + sizeof(TD)) : 0;
        if (launch_cluster(sum, blocks, 1, ring, s, a) != cudaSuccess ||
            launch(bwd_merge_kernel, (int64_t)a.B * a.G, s, a) != cudaSuccess || launch(apply, blocks, s, a) != cudaSuccess)
            return launch_failed();
    }
    if ((a.dgamma || a.dbeta) && launch(affine_grad_kernel, (a.C + AFFINE_CHANNELS - 1) / AFFINE_CHANNELS, s, a) != cudaSuccess) return launch_failed();
    return launch_status();
}

}  // namespace gn
}  // namespace minw

using namespace minw;
using namespace minw_host;

extern "C" {

minw_status minw_group_norm_backward(const void *x, int32_t x_type, int64_t ldx, const void *dy, int32_t dy_type,
                                     int64_t lddy, const float *gamma, const float *beta, const float *mean,
                                     const float *rstd, int32_t B, int64_t P, int32_t C, int32_t G, int32_t act,
                                     void *dx, int64_t lddx, float *dgamma, float *dbeta, void *workspace,
                                     size_t workspace_bytes, void *stream) {
    if ((B != 0 && (!x || !dy || !dx || !mean || !rstd)) || B < 0 || P < 1 || C < 1 || G < 1 || C % G != 0) return MINW_EINVAL;
    if (ldx < C || lddy < C || lddx < C) return MINW_EINVAL;
    if (!gn::valid_type(x_type) || !gn::valid_type(dy_type) || act < MINW_ACT_NONE || act > MINW_ACT_SILU)
        return MINW_EINVAL;
    if (!gn::fits(x, 1, x_type, 1) || !gn::fits(dy, 1, dy_type, 1) || !gn::fits(dx, 1, x_type, 1)) return MINW_EINVAL;
    if (!on_floats(gamma, beta, mean, rstd, dgamma, dbeta)) return MINW_EINVAL;
    if (!gn::in_place_ok(x, x_type, ldx, dx, x_type, lddx) || !gn::in_place_ok(dy, dy_type, lddy, dx, x_type, lddx))
        return MINW_EINVAL;
    if (P >= (1ll << 30)) return MINW_EUNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream;
    if (B == 0) {
        if (dgamma && cudaMemsetAsync(dgamma, 0, sizeof(float) * (size_t)C, s) != cudaSuccess) return launch_failed();
        if (dbeta && cudaMemsetAsync(dbeta, 0, sizeof(float) * (size_t)C, s) != cudaSuccess) return launch_failed();
        return MINW_OK;
    }
    const gn::Layout l = gn::layout(B, P, C, G, true);
    if (!workspace || !aligned16(workspace) || workspace_bytes < l.total) return MINW_EINVAL;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    gn::Args a{};
    a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy; a.y = dx; a.ldy = lddx; a.gamma = gamma; a.beta = beta;
    a.mean_in = mean; a.rstd_in = rstd; a.dgamma = dgamma; a.dbeta = dbeta;
    a.wide_affine = gamma && beta && aligned16(gamma) && aligned16(beta);
    a.B = B; a.P = (int)P; a.C = C; a.G = G; a.Cg = C / G; a.act = act;
    a.part = reinterpret_cast<float2 *>(ws + l.part);
    a.stat = reinterpret_cast<float2 *>(ws + l.stat);
    a.chan = reinterpret_cast<float2 *>(ws + l.chan);
    int V = x_type == MINW_BF16 && dy_type == MINW_BF16 ? 8 : 4;      // 16 bytes of the wider type
    while (V > 1 && (C % V != 0 || !gn::fits(x, ldx, x_type, V) || !gn::fits(dy, lddy, dy_type, V) ||
                     !gn::fits(dx, lddx, x_type, V)))
        V = V == 8 ? 4 : 1;
    if (x_type == MINW_BF16)
        return dy_type == MINW_BF16 ? gn::backward<uint16_t, uint16_t>(a, V, s)
                                    : gn::backward<uint16_t, float>(a, V, s);
    return dy_type == MINW_BF16 ? gn::backward<float, uint16_t>(a, V, s) : gn::backward<float, float>(a, V, s);
}

}  // extern "C"
