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

// GPT: groups among a thread's V channels (V / GPT channels of each).
template <typename T, typename TY, int V, int GPT, int NV>
__global__ void __launch_bounds__(THREADS) fused_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int W = V / GPT;
    __shared__ float em[THREADS * GPT], eq[THREADS * GPT];
    __shared__ float2 cta[MAX_SLAB_GROUPS], all[MAX_SLAB_GROUPS];
    const Tile w = tile<V>(a);
    const T *x = static_cast<const T *>(a.x) + ((int64_t)w.b * a.P + w.p0 + w.row) * a.ldx + w.c;
    Vec<T, V> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i < w.n) v[i].load(x + (int64_t)(i * w.rows) * a.ldx);

    // this thread's statistics of each of its groups: n W values
    const float inv = w.n > 0 ? 1.0f / (float)(w.n * W) : 0.0f;
#pragma unroll
    for (int g = 0; g < GPT; ++g) {
        float s = 0.0f, q = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < w.n) {
#pragma unroll
                for (int k = 0; k < W; ++k) s += v[i].get(g * W + k);
            }
        s *= inv;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < w.n) {
#pragma unroll
                for (int k = 0; k < W; ++k) {
                    const float d = v[i].get(g * W + k) - s;
                    q = fmaf(d, d, q);
                }
            }
        if (w.row < w.rows) {
            em[(w.row * a.L + w.lane) * GPT + g] = s;
            eq[(w.row * a.L + w.lane) * GPT + g] = q;
        }
    }
    __syncthreads();

    // a warp per group: the rows x (Cg / W) entries of this block
    const int groups = a.L * V / a.Cg, per = a.Cg / W, np = w.p1 - w.p0, lane = threadIdx.x & 31;
    for (int g = threadIdx.x >> 5; g < groups; g += THREADS / 32) {
        float s = 0.0f;
        const int entries = min(w.rows, np) * per;
        for (int e = lane; e < entries; e += 32) {
            const int r = e / per;
            s = fmaf((float)((np - r + w.rows - 1) / w.rows), em[r * a.L * GPT + g * per + e % per], s);
        }
        const float mean = np > 0 ? warp_sum(s) / ((float)np * (float)per) : 0.0f;
        s = 0.0f;
        for (int e = lane; e < entries; e += 32) {
            const int r = e / per, at = r * a.L * GPT + g * per + e % per;
            const float d = em[at] - mean;
            s += fmaf(d * d, (float)((np - r + w.rows - 1) / w.rows * W), eq[at]);
        }
        s = warp_sum(s);
        if (lane == 0) cta[g] = make_float2(mean, s);
    }

    // the cluster's blocks; the same sums in every block
    cg::cluster_group cluster = cg::this_cluster();
    if (a.chunks > 1) cluster.sync();
    else __syncthreads();
    for (int g = threadIdx.x >> 5; g < groups; g += THREADS / 32) {
        float2 t = make_float2(0.0f, 0.0f);
        float n = 0.0f;
        if (lane < a.chunks) {
            t = *(a.chunks > 1 ? cluster.map_shared_rank(&cta[g], lane) : &cta[g]);
            const int q0 = min(a.P, lane * a.ppc);
            n = (float)(min(a.P, q0 + a.ppc) - q0) * (float)a.Cg;
        }
        const float total = (float)a.P * (float)a.Cg;
        const float mean = warp_sum(n * t.x) / total;
        const float d = t.x - mean;
        const float rstd = 1.0f / sqrtf(warp_sum(n > 0.0f ? fmaf(d * d, n, t.y) : 0.0f) / total + a.eps);
        if (lane == 0) {
            all[g] = make_float2(mean, rstd);
            if (w.rank == 0) {
                const int64_t at = (int64_t)w.b * a.G + w.slab * groups + g;
                if (a.mean) a.mean[at] = mean;
                if (a.rstd) a.rstd[at] = rstd;
            }
        }
    }
    if (a.chunks > 1) cluster.barrier_arrive();
    __syncthreads();
    if (w.n > 0) {
        float ga[V], be[V], mean[GPT], rstd[GPT];
        load_affine<V>(a, w.c, ga, be);
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            const float2 t = all[(w.lane * V + g * W) / a.Cg];
            mean[g] = t.x;
            rstd[g] = t.y;
        }
        TY *y = static_cast<TY *>(a.y) + ((int64_t)w.b * a.P + w.p0 + w.row) * a.ldy + w.c;
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < w.n) {
                    float z[V];
#pragma unroll
                    for (int k = 0; k < V; ++k)
                        z[k] = act_value<act.value>(fmaf((v[i].get(k) - mean[k / W]) * rstd[k / W], ga[k], be[k]));
                    Vec<TY, V> o;
                    o.set(z);
                    o.store(y + (int64_t)(i * w.rows) * a.ldy);
                }
        });
    }
    if (a.chunks > 1) cluster.barrier_wait();              // no block leaves while its sums are read
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
                           : pl.V == 4 ? (pl.GPT == 1 ? fused_of<T, TY, 4, 1>(pl.NV) : fused_of<T, TY, 4, 4>(pl.NV))
                                       : nullptr;
        if constexpr (sizeof(T) == 2)
            if (pl.V == 8) kern = pl.GPT == 1 ? fused_of<T, TY, 8, 1>(pl.NV) : fused_of<T, TY, 8, 2>(pl.NV);
        if (launch_cluster(kern, blocks, s, f) != cudaSuccess) return MINW_ECUDA;
        return launch_status();
    }
    lanes(a, V);
    const int64_t blocks = (int64_t)a.B * a.chunks * a.slabs;
    if (blocks >= (1ll << 31) || (int64_t)a.B * a.G >= (1ll << 31)) return MINW_EUNSUPPORTED;
    void (*stat)(Args) = V == 4 ? stat_kernel<T, 4> : stat_kernel<T, 1>;
    void (*apply)(Args) = V == 4 ? apply_kernel<T, TY, 4> : apply_kernel<T, TY, 1>;
    if constexpr (sizeof(T) == 2)
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
    int V = x_type == MINW_BF16 ? 8 : 4;
    while (V > 1 && (C % V != 0 || !gn::fits(x, ldx, x_type, V) || !gn::fits(y, ldy, y_type, V))) V = V == 8 ? 4 : 1;
    cudaStream_t s = (cudaStream_t)stream;
    if (x_type == MINW_BF16)
        return y_type == MINW_BF16 ? gn::forward<uint16_t, uint16_t>(a, V, s) : gn::forward<uint16_t, float>(a, V, s);
    return y_type == MINW_BF16 ? gn::forward<float, uint16_t>(a, V, s) : gn::forward<float, float>(a, V, s);
}

}  // extern "C"
