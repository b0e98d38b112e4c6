// group_norm.cu -- group norm with an activation on channels-last rows,
// forward and backward.
//
// Statistics of n values are (count, mean, M2 = sum of squared deviations from
// that mean), and two sets merge exactly as
//   mean = (n_a m_a + n_b m_b) / (n_a + n_b),
//   M2 = M2_a + M2_b + n_a (m_a - mean)^2 + n_b (m_b - mean)^2,
// so a mean far from zero costs no digits and one pass over the data is
// enough: a thread takes the mean and M2 of the values it holds, threads,
// blocks and clusters merge in a fixed order.
//
// Both directions are bound by memory: the forward has to read x and write y,
// the backward to read x and dy and write dx.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "kernels.cuh"
#include "values.cuh"

namespace cg = cooperative_groups;

namespace minw {
namespace gn {

constexpr int THREADS = 256;

struct Args {
    const void *x, *dy;
    void *y;                       // y, or dx
    int64_t ldx, lddy, ldy;
    const float *gamma, *beta;     // nullable
    const float *mean_in, *rstd_in;
    float *mean, *rstd;            // forward: saved statistics (nullable)
    float2 *part;                  // streaming: per image, chunk and channel (mean, M2), or (sum dz, sum dz xh)
    float2 *stat;                  // streaming: per image and group (mean, rstd), or (s1, s2)
    float2 *chan;                  // backward: per image and channel (sum dz, sum dz xh)
    float *dgamma, *dbeta;         // nullable
    int B, P, C, G, Cg, act;
    float eps;
    int chunks, ppc;               // pixel chunks per image, pixels per chunk
    int L, slabs;                  // lanes (V channels each) of a slab, slabs of a row
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// gamma and beta of channels c .. c + V - 1.
template <int V>
__device__ __forceinline__ void load_affine(const Args &a, int c, float *ga, float *be) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        ga[i] = a.gamma ? a.gamma[c + i] : 1.0f;
        be[i] = a.beta ? a.beta[c + i] : 0.0f;
    }
}

// Where a block of the streaming kernels works: image, chunk of its pixels, slab of its channels.
struct Place {
    int b, chunk, slab, p0, p1, rows, row, c;
    bool active;
};
template <int V>
__device__ __forceinline__ Place place(const Args &a, int64_t block) {
    Place w;
    w.slab = (int)(block % a.slabs);
    const int64_t bc = block / a.slabs;
    w.chunk = (int)(bc % a.chunks);
    w.b = (int)(bc / a.chunks);
    w.p0 = w.chunk * a.ppc;
    w.p1 = min(a.P, w.p0 + a.ppc);
    w.rows = THREADS / a.L;
    w.row = (int)threadIdx.x / a.L;
    w.c = (w.slab * a.L + (int)threadIdx.x % a.L) * V;
    w.active = w.row < w.rows && w.c < a.C;
    return w;
}

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
                z[i] = act_value(fmaf((v[u].get(i) - mean[i]) * rstd[i], ga[i], be[i]), a.act);
            Vec<TY, V> o;
            o.set(z);
            o.store(y + (int64_t)(p + u * w.rows) * a.ldy);
        }
    }
}

// ---------------------------------------------------------------------------
// Streaming backward: the channel sums per chunk, merged per image, then a
// second pass over x and dy.
// ---------------------------------------------------------------------------

// Statistics of the V channels at c.
template <int V>
__device__ __forceinline__ void load_stats(const Args &a, int b, int c, float *mean, float *rstd) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int64_t g = (int64_t)b * a.G + (c + i) / a.Cg;
        mean[i] = a.mean_in[g];
        rstd[i] = a.rstd_in[g];
    }
}

template <typename T, typename TD, int V>
__global__ void __launch_bounds__(THREADS) bwd_sum_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int U = V == 1 ? 8 : 2;
    __shared__ float2 red[THREADS * V];
    const Place w = place<V>(a, blockIdx.x);
    float db[V], dg[V];
#pragma unroll
    for (int i = 0; i < V; ++i) db[i] = dg[i] = 0.0f;
    if (w.active) {
        float ga[V], be[V], mean[V], rstd[V];
        load_affine<V>(a, w.c, ga, be);
        load_stats<V>(a, w.b, w.c, mean, rstd);
        const T *x = static_cast<const T *>(a.x) + (int64_t)w.b * a.P * a.ldx + w.c;
        const TD *dy = static_cast<const TD *>(a.dy) + (int64_t)w.b * a.P * a.lddy + w.c;
        for (int p = w.p0 + w.row; p < w.p1; p += U * w.rows) {
            Vec<T, V> v[U];
            Vec<TD, V> d[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * w.rows < w.p1) {
                    v[u].load(x + (int64_t)(p + u * w.rows) * a.ldx);
                    d[u].load(dy + (int64_t)(p + u * w.rows) * a.lddy);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p + u * w.rows >= w.p1) break;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xh = (v[u].get(i) - mean[i]) * rstd[i];
                    const float dz = act_grad(fmaf(xh, ga[i], be[i]), d[u].get(i), a.act);
                    db[i] += dz;
                    dg[i] = fmaf(dz, xh, dg[i]);
                }
            }
        }
    }
    const int W = a.L * V;
    if (w.row < w.rows) {
#pragma unroll
        for (int i = 0; i < V; ++i) red[w.row * W + ((int)threadIdx.x % a.L) * V + i] = make_float2(db[i], dg[i]);
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
        a.part[((int64_t)w.b * a.chunks + w.chunk) * a.C + c] = make_float2(s0, s1);
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
__global__ void __launch_bounds__(THREADS) bwd_apply_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int U = V == 1 ? 8 : 2;
    const Place w = place<V>(a, (int64_t)gridDim.x - 1 - blockIdx.x);
    if (!w.active) return;
    float ga[V], be[V], mean[V], rstd[V], s1[V], s2[V];
    load_affine<V>(a, w.c, ga, be);
    load_stats<V>(a, w.b, w.c, mean, rstd);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 t = a.stat[(int64_t)w.b * a.G + (w.c + i) / a.Cg];
        s1[i] = t.x;
        s2[i] = t.y;
    }
    const T *x = static_cast<const T *>(a.x) + (int64_t)w.b * a.P * a.ldx + w.c;
    const TD *dy = static_cast<const TD *>(a.dy) + (int64_t)w.b * a.P * a.lddy + w.c;
    T *dx = static_cast<T *>(a.y) + (int64_t)w.b * a.P * a.ldy + w.c;
    for (int p = w.p0 + w.row; p < w.p1; p += U * w.rows) {
        Vec<T, V> v[U];
        Vec<TD, V> d[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * w.rows < w.p1) {
                v[u].load(x + (int64_t)(p + u * w.rows) * a.ldx);
                d[u].load(dy + (int64_t)(p + u * w.rows) * a.lddy);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * w.rows >= w.p1) break;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (v[u].get(i) - mean[i]) * rstd[i];
                const float dz = act_grad(fmaf(xh, ga[i], be[i]), d[u].get(i), a.act);
                o[i] = rstd[i] * (fmaf(ga[i], dz, -s1[i]) - xh * s2[i]);
            }
            Vec<T, V> r;
            r.set(o);
            r.store(dx + (int64_t)(p + u * w.rows) * a.ldy);
        }
    }
}

// dbeta, dgamma: the images' channel sums, a warp per channel of 32, 8 rows of images side by side.
__global__ void __launch_bounds__(THREADS) affine_grad_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    __shared__ float2 red[8][33];
    const int c = (int)blockIdx.x * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
    float db = 0.0f, dg = 0.0f;
    if (c < a.C)
        for (int b = r; b < a.B; b += 8) {
            const float2 t = a.chan[(int64_t)b * a.C + c];
            db += t.x;
            dg += t.y;
        }
    red[r][threadIdx.x & 31] = make_float2(db, dg);
    __syncthreads();
    if (r == 0 && c < a.C) {
        db = dg = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            db += red[k][threadIdx.x].x;
            dg += red[k][threadIdx.x].y;
        }
        if (a.dbeta) a.dbeta[c] = db;
        if (a.dgamma) a.dgamma[c] = dg;
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

using namespace minw_host;

static size_t al256(size_t v) { return (v + 255) & ~(size_t)255; }

// Pixel chunks per image of the streaming kernels: about eight blocks per SM over all images, at least 64 pixels each.
static int chunks_of(int B, int64_t P) {
    int64_t k = (8 * 152 + B - 1) / B;
    if (k > (P + 63) / 64) k = (P + 63) / 64;
    return (int)(k < 1 ? 1 : k);
}

struct Layout {
    size_t part, stat, chan, total;
};
static Layout layout(int B, int64_t P, int C, int G, bool backward) {
    Layout l;
    size_t off = 0;
    auto take = [&](size_t n) { const size_t r = off; off += al256(n * sizeof(float2)); return r; };
    l.part = take((size_t)B * chunks_of(B, P) * C);
    l.stat = take((size_t)B * G);
    l.chan = backward ? take((size_t)B * C) : off;
    l.total = off;
    return l;
}

static bool valid_type(int t) { return t == MINW_F32 || t == MINW_BF16; }
static int bytes_of(int t) { return t == MINW_BF16 ? 2 : 4; }

// Whether a tensor's rows start on multiples of V values (at most 16 bytes of them).
static bool fits(const void *p, int64_t ld, int type, int V) {
    const int bytes = bytes_of(type) * V > 16 ? 16 : bytes_of(type) * V;
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * bytes_of(type) % bytes == 0;
}

// An output at an input's address replaces it value by value.
static bool in_place_ok(const void *in, int in_type, int64_t in_ld, const void *out, int out_type, int64_t out_ld) {
    return in == nullptr || in != out || (in_type == out_type && in_ld == out_ld);
}

static cudaError_t launch(void (*kern)(Args), int64_t blocks, cudaStream_t s, const Args &a) {
    return launch_pdl_stream(false, kern, dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
}

// Lanes and slabs of the streaming kernels for V channels a lane.
static void lanes(Args &a, int V) {
    const int lanes = a.C / V;
    a.slabs = (lanes + THREADS - 1) / THREADS;
    a.L = (lanes + a.slabs - 1) / a.slabs;
}

template <typename T, typename TY>
static minw_status forward(Args a, int V, cudaStream_t s) {
    lanes(a, V);
    const int64_t blocks = (int64_t)a.B * a.chunks * a.slabs;
    if (blocks >= (1ll << 31) || (int64_t)a.B * a.G >= (1ll << 31)) return MINW_EUNSUPPORTED;
    auto stat = V == 8 ? stat_kernel<T, 8> : V == 4 ? stat_kernel<T, 4> : stat_kernel<T, 1>;
    auto apply = V == 8 ? apply_kernel<T, TY, 8> : V == 4 ? apply_kernel<T, TY, 4> : apply_kernel<T, TY, 1>;
    if (launch(stat, blocks, s, a) != cudaSuccess || launch(stat_merge_kernel, (int64_t)a.B * a.G, s, a) != cudaSuccess ||
        launch(apply, blocks, s, a) != cudaSuccess)
        return MINW_ECUDA;
    return launch_status();
}

template <typename T, typename TD>
static minw_status backward(Args a, int V, cudaStream_t s) {
    lanes(a, V);
    const int64_t blocks = (int64_t)a.B * a.chunks * a.slabs;
    if (blocks >= (1ll << 31) || (int64_t)a.B * a.G >= (1ll << 31)) return MINW_EUNSUPPORTED;
    auto sum = V == 8 ? bwd_sum_kernel<T, TD, 8> : V == 4 ? bwd_sum_kernel<T, TD, 4> : bwd_sum_kernel<T, TD, 1>;
    auto apply = V == 8 ? bwd_apply_kernel<T, TD, 8> : V == 4 ? bwd_apply_kernel<T, TD, 4> : bwd_apply_kernel<T, TD, 1>;
    if (launch(sum, blocks, s, a) != cudaSuccess || launch(bwd_merge_kernel, (int64_t)a.B * a.G, s, a) != cudaSuccess ||
        launch(apply, blocks, s, a) != cudaSuccess)
        return MINW_ECUDA;
    if ((a.dgamma || a.dbeta) && launch(affine_grad_kernel, (a.C + 31) / 32, s, a) != cudaSuccess) return MINW_ECUDA;
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
    if (!gn::in_place_ok(x, x_type, ldx, dx, x_type, lddx) || !gn::in_place_ok(dy, dy_type, lddy, dx, x_type, lddx))
        return MINW_EINVAL;
    if (P >= (1ll << 30)) return MINW_EUNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream;
    if (B == 0) {
        if (dgamma && cudaMemsetAsync(dgamma, 0, sizeof(float) * (size_t)C, s) != cudaSuccess) return MINW_ECUDA;
        if (dbeta && cudaMemsetAsync(dbeta, 0, sizeof(float) * (size_t)C, s) != cudaSuccess) return MINW_ECUDA;
        return MINW_OK;
    }
    const gn::Layout l = gn::layout(B, P, C, G, true);
    if (!workspace || !aligned16(workspace) || workspace_bytes < l.total) return MINW_EINVAL;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    gn::Args a{};
    a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy; a.y = dx; a.ldy = lddx; a.gamma = gamma; a.beta = beta;
    a.mean_in = mean; a.rstd_in = rstd; a.dgamma = dgamma; a.dbeta = dbeta;
    a.B = B; a.P = (int)P; a.C = C; a.G = G; a.Cg = C / G; a.act = act;
    a.chunks = gn::chunks_of(B, P);
    a.ppc = (int)((P + a.chunks - 1) / a.chunks);
    a.chunks = (int)((P + a.ppc - 1) / a.ppc);
    a.part = reinterpret_cast<float2 *>(ws + l.part);
    a.stat = reinterpret_cast<float2 *>(ws + l.stat);
    a.chan = reinterpret_cast<float2 *>(ws + l.chan);
    int V = x_type == MINW_BF16 ? 8 : 4;
    while (V > 1 && (C % V != 0 || !gn::fits(x, ldx, x_type, V) || !gn::fits(dy, lddy, dy_type, V) ||
                     !gn::fits(dx, lddx, x_type, V)))
        V = V == 8 ? 4 : 1;
    if (x_type == MINW_BF16)
        return dy_type == MINW_BF16 ? gn::backward<uint16_t, uint16_t>(a, V, s)
                                    : gn::backward<uint16_t, float>(a, V, s);
    return dy_type == MINW_BF16 ? gn::backward<float, uint16_t>(a, V, s) : gn::backward<float, float>(a, V, s);
}

}  // extern "C"
