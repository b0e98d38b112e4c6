// group_norm.cu -- forward of the group norm with an activation on
// channels-last rows (group_norm.cuh: statistics, tiles and plans).
#include "group_norm.cuh"

namespace minw {
namespace gn {

// ---------------------------------------------------------------------------
// Streaming forward: statistics per chunk and channel, merged per group, then
// a second pass over x.
// ---------------------------------------------------------------------------

template <typename T, int V>
__global__ void __launch_bounds__(THREADS) stat_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int U = V == 1 ? 8 : 4;                        // pixels in flight per thread
    __shared__ float2 red[THREADS * V];
    const Place w = place<V>(a, blockIdx.x);
    float m[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) m[i] = q[i] = 0.0f;
    int n = 0;
    if (w.active) {
        const T *x = static_cast<const T *>(a.x) + (int64_t)w.b * a.P * a.ldx + w.c;
        for (int p = w.p0 + w.row; p < w.p1; p += U * w.rows) {
            Vec<T, V> v[U];
            int k = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * w.rows < w.p1) {
                    v[u].load(x + (int64_t)(p + u * w.rows) * a.ldx);
                    k = u + 1;
                }
            const float inv = 1.0f / (float)k, share = (float)k / (float)(n + k);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float s = 0.0f, d2 = 0.0f;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u < k) s += v[u].get(i);
                s *= inv;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u < k) {
                        const float d = v[u].get(i) - s;
                        d2 = fmaf(d, d, d2);
                    }
                const float d = s - m[i];
                m[i] = fmaf(d, share, m[i]);
                q[i] += fmaf(d * d, (float)n * share, d2);
            }
            n += k;
        }
    }
    // rows of the block: row r holds (pixels - r + rows - 1) / rows of them
    const int W = a.L * V, np = w.p1 - w.p0;
    if (w.row < w.rows) {
#pragma unroll
        for (int i = 0; i < V; ++i) red[w.row * W + ((int)threadIdx.x % a.L) * V + i] = make_float2(m[i], q[i]);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < W; e += THREADS) {
        const int c = w.slab * W + e;
        if (c >= a.C) break;
        float s = 0.0f;
        for (int r = 0; r < w.rows; ++r) s = fmaf((float)((np - r + w.rows - 1) / w.rows), red[r * W + e].x, s);
        const float mean = s / (float)np;
        float M2 = 0.0f;
        for (int r = 0; r < w.rows; ++r) {
            const float2 t = red[r * W + e];
            const float d = t.x - mean;
            M2 += fmaf(d * d, (float)((np - r + w.rows - 1) / w.rows), t.y);
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
    for (int e = threadIdx.x; e < entries; e += THREADS) {
        const int k = e / a.Cg;
        s = fmaf((float)(min(a.P, (k + 1) * a.ppc) - k * a.ppc), part[(int64_t)k * a.C + e % a.Cg].x, s);
    }
    const float mean = block_sum(s) / n;
    s = 0.0f;
    for (int e = threadIdx.x; e < entries; e += THREADS) {
        const int k = e / a.Cg;
        const float2 t = part[(int64_t)k * a.C + e % a.Cg];
        const float d = t.x - mean;
        s += fmaf(d * d, (float)(min(a.P, (k + 1) * a.ppc) - k * a.ppc), t.y);
    }
    const float rstd = 1.0f / sqrtf(block_sum(s) / n + a.eps);
    if (threadIdx.x == 0) {
        a.stat[blockIdx.x] = make_float2(mean, rstd);
        if (a.mean) a.mean[blockIdx.x] = mean;
        if (a.rstd) a.rstd[blockIdx.x] = rstd;
    }
}

template <typename T, typename TY, int V>
__global__ void __launch_bounds__(THREADS) apply_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int U = V == 1 ? 8 : 4;
    const Place w = place<V>(a, (int64_t)gridDim.x - 1 - blockIdx.x);     // the last chunks read are still in L2
    if (!w.active) return;
    float ga[V], be[V], mean[V], rstd[V];
    load_affine<V>(a, w.c, ga, be);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 t = a.stat[(int64_t)w.b * a.G + (w.c + i) / a.Cg];
        mean[i] = t.x;
        rstd[i] = t.y;
    }
    const T *x = static_cast<const T *>(a.x) + (int64_t)w.b * a.P * a.ldx + w.c;
    TY *y = static_cast<TY *>(a.y) + (int64_t)w.b * a.P * a.ldy + w.c;
    with_act(a.act, [&](auto act) {
        for (int p = w.p0 + w.row; p < w.p1; p += U * w.rows) {
            Vec<T, V> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * w.rows < w.p1) v[u].load(x + (int64_t)(p + u * w.rows) * a.ldx);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p + u * w.rows >= w.p1) break;
                float z[V];
#pragma unroll
                for (int i = 0; i < V; ++i)
                    z[i] = act_value<act.value>(fmaf((v[u].get(i) - mean[i]) * rstd[i], ga[i], be[i]));
                Vec<TY, V> o;
                o.set(z);
                o.store(y + (int64_t)(p + u * w.rows) * a.ldy);
            }
        }
    });
}

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

// GPT: groups among a thread's V channels (W = V / GPT channels of each).  A thread sums its values and their
// squared deviations from its own mean; the block's mean turns the latter into deviations from that (n W (m - mean)^2
// more), and the cluster's mean likewise.
template <typename T, typename TY, int V, int GPT, int NV>
__global__ void __launch_bounds__(THREADS, NV == 8 ? 4 : NV == 16 ? 2 : 3) fused_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int W = V / GPT, NP = (V + 1) / 2;
    __shared__ GroupSum<GPT> sums[2];
    __shared__ float2 cta[MAX_SLAB_GROUPS], all[MAX_SLAB_GROUPS];
    const Tile w = tile<V>(a);
    const T *x = static_cast<const T *>(a.x) + ((int64_t)w.b * a.P + w.p0 + w.row) * a.ldx + w.c;
    const int64_t step = (int64_t)w.rows * a.ldx;
    Vec<T, V> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i < w.n) v[i].load(x + i * step);

    float mean[GPT], m2[GPT];
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
        auto fold = [&](const Pair *p, float *f) {
            if constexpr (W == 1) {
#pragma unroll
                for (int k = 0; k < NP; ++k) {
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
        };
        fold(s, mean);
        const float values = (float)(w.n * W), inv = w.n > 0 ? __fdividef(1.0f, values) : 0.0f;
        float own[GPT];
#pragma unroll
        for (int g = 0; g < GPT; ++g) own[g] = mean[g] * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < w.n) {
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    const Pair d = add2(v[i].get2(k), pick_group<V, W>(own, k, -1.0f));
                    q[k] = fma2(d, d, q[k]);
                }
            }
        fold(q, m2);
        group_sum<GPT>(mean, sums[0], a, w);
        const float block = w.p1 > w.p0 ? __fdividef(1.0f, (float)(w.p1 - w.p0) * (float)a.Cg) : 0.0f;
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            mean[g] *= block;
            const float d = own[g] - mean[g];
            if (w.n > 0) m2[g] = fmaf(d * d, values, m2[g]);
        }
        group_sum<GPT>(m2, sums[1], a, w);
    }

    float rstd[GPT];
    if (a.chunks > 1) {
        // the cluster's blocks: sixteen threads a group, one for each; the same sums in every block
        if (w.row == 0) {
#pragma unroll
            for (int g = 0; g < GPT; ++g) cta[a.by_per.div(w.lane * GPT + g)] = make_float2(mean[g], m2[g]);
        }
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        for (int g = threadIdx.x >> 4; g < (a.groups + 1) / 2 * 2; g += THREADS / 16) {    // both halves of a warp alike
            const int k = threadIdx.x & 15;
            float2 t = make_float2(0.0f, 0.0f);
            float n = 0.0f;
            if (k < a.chunks && g < a.groups) {
                t = *cluster.map_shared_rank(&cta[g], k);
                const int q0 = min(a.P, k * a.ppc);
                n = (float)(min(a.P, q0 + a.ppc) - q0) * (float)a.Cg;
            }
            float s = n * t.x;
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
            s *= a.inv_total;
            const float d0 = t.x - s;
            float q = n > 0.0f ? fmaf(d0 * d0, n, t.y) : 0.0f;
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) q += __shfl_xor_sync(0xffffffffu, q, d);
            if (k == 0 && g < a.groups) all[g] = make_float2(s, q);
        }
        cluster_done_reading();
        __syncthreads();
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            const float2 t = all[a.by_per.div(w.lane * GPT + g)];
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
    if (w.n > 0) {
        float ga[V], be[V];
        load_affine<V>(a, w.c, ga, be);
        TY *y = static_cast<TY *>(a.y) + ((int64_t)w.b * a.P + w.p0 + w.row) * a.ldy + w.c;
        const int64_t ystep = (int64_t)w.rows * a.ldy;
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < w.n) {
                    float z[2 * NP];
#pragma unroll
                    for (int k = 0; k < NP; ++k) {
                        const Pair xh = mul2(add2(v[i].get2(k), pick_group<V, W>(mean, k, -1.0f)), pick_group<V, W>(rstd, k));
                        const float2 h = halves(fma2(xh, pick<V>(ga, k), pick<V>(be, k)));
                        z[2 * k] = act_value<act.value>(h.x);
                        z[2 * k + 1] = act_value<act.value>(h.y);
                    }
                    Vec<TY, V> o;
                    o.set(z);
                    o.store(y + i * ystep);
                }
        });
    }
    if (a.chunks > 1) cluster_leave();
}

template <typename T, typename TY, int V, int GPT>
static auto fused_of(int NV) {
    if constexpr (V == 1) return fused_kernel<T, TY, 1, 1, 32>;
    else return NV == 8 ? fused_kernel<T, TY, V, GPT, 8> : fused_kernel<T, TY, V, GPT, 16>;
}
template <typename T, typename TY>
static minw_status forward(Args a, int V, cudaStream_t s) {
    Plan pl;
    if (Args f = a; one_pass(f, pl, (int)sizeof(T), V, false)) {
        const int64_t blocks = (int64_t)f.B * f.slabs * f.chunks;
        if (blocks >= (1ll << 31)) return MINW_EUNSUPPORTED;
        void (*kern)(Args) = pl.V == 1 ? fused_of<T, TY, 1, 1>(pl.NV)
                           : pl.V == 4 ? (pl.GPT == 1 ? fused_of<T, TY, 4, 1>(pl.NV) : pl.GPT == 2 ? fused_of<T, TY, 4, 2>(pl.NV)
                                                                                       : fused_of<T, TY, 4, 4>(pl.NV))
                                       : nullptr;
        if constexpr (sizeof(T) == 2 && sizeof(TY) == 2)
            if (pl.V == 8)
                kern = pl.GPT == 1   ? fused_of<T, TY, 8, 1>(pl.NV)
                       : pl.GPT == 2 ? fused_of<T, TY, 8, 2>(pl.NV)
                                     : fused_of<T, TY, 8, 4>(pl.NV);
        if (launch_cluster(kern, blocks, s, f) != cudaSuccess) return MINW_ECUDA;
        return launch_status();
    }
    lanes(a, V);
    const int64_t blocks = (int64_t)a.B * a.chunks * a.slabs;
    if (blocks >= (1ll << 31) || (int64_t)a.B * a.G >= (1ll << 31)) return MINW_EUNSUPPORTED;
    void (*stat)(Args) = V == 4 ? stat_kernel<T, 4> : stat_kernel<T, 1>;
    void (*apply)(Args) = V == 4 ? apply_kernel<T, TY, 4> : apply_kernel<T, TY, 1>;
    if constexpr (sizeof(T) == 2 && sizeof(TY) == 2)
        if (V == 8) {
            stat = stat_kernel<T, 8>;
            apply = apply_kernel<T, TY, 8>;
        }
    if (launch(stat, blocks, s, a) != cudaSuccess || launch(stat_merge_kernel, (int64_t)a.B * a.G, s, a) != cudaSuccess ||
        launch(apply, blocks, s, a) != cudaSuccess)
        return MINW_ECUDA;
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
    if (P >= (1ll << 30)) return MINW_EUNSUPPORTED;
    if (B == 0) return MINW_OK;
    const gn::Layout l = gn::layout(B, P, C, G, false);
    if (!workspace || !aligned16(workspace) || workspace_bytes < l.total) return MINW_EINVAL;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    gn::Args a{};
    a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy; a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd;
    a.B = B; a.P = (int)P; a.C = C; a.G = G; a.Cg = C / G; a.act = act; a.eps = eps;
    a.chunks = gn::chunks_of(B, P);
    a.ppc = (int)((P + a.chunks - 1) / a.chunks);
    a.chunks = (int)((P + a.ppc - 1) / a.ppc);                // no chunk without a pixel
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
