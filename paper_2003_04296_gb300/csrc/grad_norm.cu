// grad_norm.cu -- the global norm of a network's gradients, clipping by it, and
// the clipped update of Algorithm 1, over lists of tensors.
//
// Two kernels: the first sums the squares, a partial sum per block; every block
// of the second adds the partial sums up again (a few kilobytes from L2, in the
// same order everywhere) and then scales or updates its share.  The tensors'
// addresses and lengths travel as kernel arguments, so a call leaves nothing
// on the device but the partial sums in the caller's workspace.
//
// Bound by memory: the gradients are read by the first kernel and again by the
// second, which takes the chunks in the opposite order so that what the L2
// still holds is read first.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "kernels.cuh"
#include "values.cuh"

namespace minw {
namespace gradn {

constexpr int THREADS = 256;
constexpr int MAX_CHUNK = 32768;     // values of a chunk at most: a thread adds 128 squares in fp32
constexpr int MAX_BLOCKS = 2048;     // partial sums of a launch at most
constexpr int CAP_MAX = 800;         // tensors of a launch: 800 x 40 bytes of the 32764 that a launch may pass

enum Op { CLIP = 0, UPDATE = 1 };

struct Entry {
    const void *g;
    void *o;              // clipped gradient, or weights
    int64_t n;
    uint32_t first;       // first chunk of this tensor
    uint16_t head;        // values before the first vector
    uint8_t g_bf16, o_bf16;
    float limit;
    uint32_t vec;         // whether both tensors' vectors are aligned after the head
};

template <int CAP>
struct List {
    Entry e[CAP];
    int count;
    uint32_t chunks;
    int chunk;            // values of a chunk (a multiple of 8 THREADS)
};

// Tensor of a chunk: the last whose first chunk is not past it.
template <int CAP>
__device__ __forceinline__ int tensor_of(const List<CAP> &l, uint32_t c) {
    int lo = 0, hi = l.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.e[mid].first <= c) lo = mid; else hi = mid;
    }
    return lo;
}

// Values [i0, i1) of a tensor's chunk k: the first chunk has the head too.
__device__ __forceinline__ void range_of(const Entry &e, uint32_t k, int chunk, int64_t &i0, int64_t &i1) {
    i0 = k == 0 ? 0 : e.head + (int64_t)k * chunk;
    i1 = e.head + (int64_t)(k + 1) * chunk;
    if (i1 > e.n) i1 = e.n;
}

__device__ __forceinline__ double block_sum(double v, double *red) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) v += red[k];
    __syncthreads();
    return v;
}

// Sum of squares of this thread's values of a chunk.
template <typename T>
__device__ __forceinline__ double chunk_squares(const T *g, int64_t i0, int64_t i1, int head) {
    constexpr int V = 16 / sizeof(T), U = 4;
    const int64_t v0 = i0 == 0 ? head : i0;                    // first aligned value
    const int64_t nv = i1 > v0 ? (i1 - v0) / V : 0, tail = v0 + nv * V;
    float s0 = 0.0f, s1 = 0.0f;
    uint32_t bits = 0;
    for (int64_t k = threadIdx.x; k < nv; k += U * THREADS) {
        Vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k + u * THREADS < nv) v[u].load(g + v0 + (k + u * THREADS) * V);
            else
                for (int w = 0; w < Vec<T, V>::WORDS; ++w) v[u].w[w] = 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int w = 0; w < Vec<T, V>::WORDS; ++w) bits |= v[u].w[w];
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                s0 = fmaf(v[u].get(i), v[u].get(i), s0);
                s1 = fmaf(v[u].get(i + 1), v[u].get(i + 1), s1);
            }
        }
    }
    auto scalar = [&](int64_t i) {
        Vec<T, 1> v;
        v.load(g + i);
        bits |= v.w[0];
        return v.get(0);
    };
    const int64_t h1 = v0 < i1 ? v0 : i1;
    for (int64_t i = i0 + threadIdx.x; i < h1; i += THREADS) { const float v = scalar(i); s0 = fmaf(v, v, s0); }
    for (int64_t i = (tail > h1 ? tail : h1) + threadIdx.x; i < i1; i += THREADS) { const float v = scalar(i); s1 = fmaf(v, v, s1); }
    const float s = s0 + s1;
    // squares below 2^-126 lose digits and above 2^128 overflow: outside these limits (the sum of at most a few
    // hundred squares is then right to fp32 precision) and unless all values are zero, the sum is taken in fp64
    if ((s >= 1e-28f && s <= 3e38f) || (bits & (sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu)) == 0u) return (double)s;
    double d = 0.0;
    for (int64_t k = threadIdx.x; k < nv; k += THREADS)
        for (int i = 0; i < V; ++i) {
            const double v = scalar(v0 + k * V + i);
            d = fma(v, v, d);
        }
    for (int64_t i = i0 + threadIdx.x; i < h1; i += THREADS) { const double v = scalar(i); d = fma(v, v, d); }
    for (int64_t i = (tail > h1 ? tail : h1) + threadIdx.x; i < i1; i += THREADS) { const double v = scalar(i); d = fma(v, v, d); }
    return d;
}

template <int CAP>
__global__ void __launch_bounds__(THREADS) squares_kernel(const __grid_constant__ List<CAP> l, double *part) {
    pdl_trigger();
    pdl_wait();
    __shared__ double red[THREADS / 32];
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
        const Entry &e = l.e[tensor_of(l, c)];
        int64_t i0, i1;
        range_of(e, c - e.first, l.chunk, i0, i1);
        s += e.g_bf16 ? chunk_squares(static_cast<const uint16_t *>(e.g), i0, i1, e.head)
                      : chunk_squares(static_cast<const float *>(e.g), i0, i1, e.head);
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm from the partial sums, by every block alike.
__device__ __forceinline__ double norm_of(const double *part, int parts, double *red) {
    double s = 0.0;
    for (int k = threadIdx.x; k < parts; k += THREADS) s += part[k];
    return sqrt(block_sum(s, red));
}

__global__ void __launch_bounds__(THREADS) norm_kernel(const double *part, int parts, float *norm) {
    pdl_trigger();
    pdl_wait();
    __shared__ double red[THREADS / 32];
    const double n = norm_of(part, parts, red);
    if (threadIdx.x == 0) *norm = (float)n;
}

template <int OP>
__device__ __forceinline__ float step(float g, float w, float k, float lr, float limit) {
    if (OP == CLIP) return k * g;
    const float v = fmaf(-lr, k * g, w);
    return v > limit ? limit : v < -limit ? -limit : v;
}

template <int OP, typename TG, typename TO>
__device__ __forceinline__ void chunk_step(const Entry &e, int64_t i0, int64_t i1, float k, float lr) {
    constexpr int V = sizeof(TG) == 2 && sizeof(TO) == 2 ? 8 : 4, U = 4;
    const TG *g = static_cast<const TG *>(e.g);
    TO *o = static_cast<TO *>(e.o);
    const int64_t v0 = i0 == 0 ? e.head : i0;
    const int64_t nv = e.vec && i1 > v0 ? (i1 - v0) / V : 0, tail = nv > 0 ? v0 + nv * V : i0;
    for (int64_t j = threadIdx.x; j < nv; j += U * THREADS) {
        Vec<TG, V> vg[U];
        Vec<TO, V> vo[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u * THREADS < nv) {
                vg[u].load(g + v0 + (j + u * THREADS) * V);
                if (OP == UPDATE) vo[u].load(o + v0 + (j + u * THREADS) * V);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j + u * THREADS >= nv) break;
            float r[V];
#pragma unroll
            for (int i = 0; i < V; ++i) r[i] = step<OP>(vg[u].get(i), OP == UPDATE ? vo[u].get(i) : 0.0f, k, lr, e.limit);
            vo[u].set(r);
            vo[u].store(o + v0 + (j + u * THREADS) * V);
        }
    }
    auto scalar = [&](int64_t i) {
        Vec<TG, 1> vg;
        Vec<TO, 1> vo;
        vg.load(g + i);
        if (OP == UPDATE) vo.load(o + i);
        const float r = step<OP>(vg.get(0), OP == UPDATE ? vo.get(0) : 0.0f, k, lr, e.limit);
        vo.set(&r);
        vo.store(o + i);
    };
    if (nv > 0)
        for (int64_t i = i0 + threadIdx.x; i < v0; i += THREADS) scalar(i);
    for (int64_t i = tail + threadIdx.x; i < i1; i += THREADS) scalar(i);
}

template <int OP, int CAP>
__global__ void __launch_bounds__(THREADS) step_kernel(const __grid_constant__ List<CAP> l, const double *part,
                                                       int parts, float max_norm, float lr, float *norm) {
    pdl_trigger();
    pdl_wait();
    __shared__ double red[THREADS / 32];
    const double n = norm_of(part, parts, red);
    const float nf = (float)n;
    if (norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *norm = nf;
    const bool finite = nf <= 3.402823466e38f;                    // false for NaN
    if (OP == UPDATE && !finite) return;
    const float k = finite && n > (double)max_norm ? (float)((double)max_norm / n) : 1.0f;
    for (uint32_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
        const uint32_t r = l.chunks - 1 - c;
        const Entry &e = l.e[tensor_of(l, r)];
        if (OP == CLIP && k == 1.0f && e.o == e.g) continue;
        int64_t i0, i1;
        range_of(e, r - e.first, l.chunk, i0, i1);
        if (OP == CLIP) {
            if (e.g_bf16) chunk_step<OP, uint16_t, uint16_t>(e, i0, i1, k, lr);
            else chunk_step<OP, float, float>(e, i0, i1, k, lr);
        } else if (e.o_bf16) {
            if (e.g_bf16) chunk_step<OP, uint16_t, uint16_t>(e, i0, i1, k, lr);
            else chunk_step<OP, float, uint16_t>(e, i0, i1, k, lr);
        } else {
            if (e.g_bf16) chunk_step<OP, uint16_t, float>(e, i0, i1, k, lr);
            else chunk_step<OP, float, float>(e, i0, i1, k, lr);
        }
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

using namespace minw_host;

static int size_of(int type) { return type == MINW_BF16 ? 2 : 4; }

static bool valid_list(const minw_tensor *l, int count) {
    for (int t = 0; t < count; ++t) {
        if (l[t].type != MINW_F32 && l[t].type != MINW_BF16) return false;
        if (l[t].n < 0 || (l[t].n > 0 && l[t].data == nullptr)) return false;
        if (reinterpret_cast<uintptr_t>(l[t].data) % size_of(l[t].type) != 0) return false;
    }
    return true;
}

// Values of a chunk: small sets are spread over the SMs, four chunks each, large ones take the longest.
static int chunk_of(int64_t total) {
    int64_t c = total / (4 * 152);
    c = (c + 8 * THREADS - 1) / (8 * THREADS) * (8 * THREADS);
    return (int)(c < 8 * THREADS ? 8 * THREADS : c > MAX_CHUNK ? MAX_CHUNK : c);
}

// Fills one launch's list from tensor t on; returns the next launch's first tensor.
template <int CAP>
static int fill(List<CAP> &l, const minw_tensor *g, const minw_tensor *o, int t, int count, int chunk) {
    l.count = 0;
    l.chunks = 0;
    l.chunk = chunk;
    for (; t < count && l.count < CAP; ++t) {
        if (g[t].n == 0) continue;
        Entry e{};
        const int gs = size_of(g[t].type), os = o ? size_of(o[t].type) : 16;
        e.g = g[t].data;
        e.o = o ? o[t].data : nullptr;
        e.n = g[t].n;
        e.g_bf16 = g[t].type == MINW_BF16;
        e.o_bf16 = o && o[t].type == MINW_BF16;
        e.limit = o ? o[t].limit : 0.0f;
        e.first = l.chunks;
        // the head ends where the gradient's 16-byte vectors begin; the other tensor's have to begin there too
        const uintptr_t ga = reinterpret_cast<uintptr_t>(e.g);
        e.head = (uint16_t)((16 - ga % 16) % 16 / gs);
        const int V = gs == 2 && os == 2 ? 8 : 4;
        e.vec = o && (reinterpret_cast<uintptr_t>(e.o) + (uintptr_t)e.head * os) % (V * os) == 0;
        const int64_t body = e.n - e.head;
        l.chunks += body > 0 ? (uint32_t)((body + chunk - 1) / chunk) : 1u;
        l.e[l.count++] = e;
    }
    return t;
}

static int blocks_of(uint32_t chunks) {
    const int sms = num_sms() > 0 ? num_sms() : 152;
    const uint32_t cap = (uint32_t)(sms * 8 < MAX_BLOCKS ? sms * 8 : MAX_BLOCKS);
    return (int)(chunks < cap ? chunks : cap);
}

struct Call {
    const minw_tensor *g, *o;
    int count, op;               // op -1: the norm alone
    float max_norm, lr;
    float *norm;
    double *part;
    cudaStream_t s;
};

template <int CAP>
static minw_status run(const Call &c, int chunk) {
    static thread_local List<CAP> l;
    int parts = 0;
    for (int t = 0; t < c.count;) {
        t = fill(l, c.g, c.o, t, c.count, chunk);
        if (l.chunks == 0) continue;
        const int blocks = blocks_of(l.chunks);
        if (launch_pdl_stream(false, squares_kernel<CAP>, dim3((unsigned)blocks), dim3(THREADS), 0, c.s, l,
                              c.part + parts) != cudaSuccess)
            return MINW_ECUDA;
        parts += blocks;
    }
    if (c.op < 0 || parts == 0) {
        if (launch_pdl_stream(false, norm_kernel, dim3(1), dim3(THREADS), 0, c.s, (const double *)c.part, parts,
                              c.norm) != cudaSuccess)
            return MINW_ECUDA;
        return launch_status();
    }
    float *norm = c.norm;
    for (int t = 0; t < c.count;) {
        t = fill(l, c.g, c.o, t, c.count, chunk);
        if (l.chunks == 0) continue;
        if (launch_pdl_stream(false, c.op == CLIP ? step_kernel<CLIP, CAP> : step_kernel<UPDATE, CAP>,
                              dim3((unsigned)blocks_of(l.chunks)), dim3(THREADS), 0, c.s, l, (const double *)c.part,
                              parts, c.max_norm, c.lr, norm) != cudaSuccess)
            return MINW_ECUDA;
        norm = nullptr;
    }
    return launch_status();
}

static minw_status check(const minw_tensor *g, const minw_tensor *o, int count, const float *norm, const void *ws,
                         size_t ws_bytes, bool same_types, int64_t &total) {
    if (count < 0 || (count > 0 && !g) || !norm || !ws) return MINW_EINVAL;
    if (!aligned16(ws) || ws_bytes < minw_grad_workspace_bytes(count)) return MINW_EINVAL;
    if (reinterpret_cast<uintptr_t>(norm) % 4 != 0) return MINW_EINVAL;
    if (!valid_list(g, count) || (o && !valid_list(o, count))) return MINW_EINVAL;
    total = 0;
    for (int t = 0; t < count; ++t) {
        if (o && (o[t].n != g[t].n || (same_types && o[t].type != g[t].type))) return MINW_EINVAL;
        if (g[t].n >= (1ll << 46) || (total += g[t].n) >= (1ll << 46)) return MINW_EUNSUPPORTED;
    }
    return MINW_OK;
}

// The list's capacity decides how many bytes of arguments a launch carries.
static minw_status dispatch(const Call &c, int64_t total) {
    const int chunk = chunk_of(total);
    return c.count <= 16 ? run<16>(c, chunk) : c.count <= 128 ? run<128>(c, chunk) : run<CAP_MAX>(c, chunk);
}

}  // namespace gradn
}  // namespace minw

using namespace minw;
using namespace minw_host;

extern "C" {

size_t minw_grad_workspace_bytes(int32_t count) {
    if (count < 0) return 0;
    const size_t launches = count <= gradn::CAP_MAX ? 1 : ((size_t)count + gradn::CAP_MAX - 1) / gradn::CAP_MAX;
    return launches * gradn::MAX_BLOCKS * sizeof(double);
}

minw_status minw_grad_norm(const minw_tensor *grads, int32_t count, float *norm, void *workspace,
                           size_t workspace_bytes, void *stream) {
    int64_t total;
    const minw_status st = gradn::check(grads, nullptr, count, norm, workspace, workspace_bytes, false, total);
    if (st != MINW_OK) return st;
    return gradn::dispatch({grads, nullptr, count, -1, 0.0f, 0.0f, norm, static_cast<double *>(workspace),
                            (cudaStream_t)stream}, total);
}

minw_status minw_grad_clip(const minw_tensor *grads, const minw_tensor *out, int32_t count, float max_norm, float *norm,
                           void *workspace, size_t workspace_bytes, void *stream) {
    if (count > 0 && !out) return MINW_EINVAL;
    if (!(max_norm > 0.0f && isfinite(max_norm))) return MINW_EINVAL;
    int64_t total;
    const minw_status st = gradn::check(grads, out, count, norm, workspace, workspace_bytes, true, total);
    if (st != MINW_OK) return st;
    return gradn::dispatch({grads, out, count, gradn::CLIP, max_norm, 0.0f, norm, static_cast<double *>(workspace),
                            (cudaStream_t)stream}, total);
}

minw_status minw_sgd_clip_norm(const minw_tensor *weights, const minw_tensor *grads, int32_t count, float max_norm,
                               float lr, float *norm, void *workspace, size_t workspace_bytes, void *stream) {
    if (count > 0 && !weights) return MINW_EINVAL;
    if (!(max_norm > 0.0f && isfinite(max_norm)) || !isfinite(lr)) return MINW_EINVAL;
    int64_t total;
    const minw_status st = gradn::check(grads, weights, count, norm, workspace, workspace_bytes, false, total);
    if (st != MINW_OK) return st;
    for (int t = 0; t < count; ++t)
        if (!(weights[t].limit >= 0.0f)) return MINW_EINVAL;
    return gradn::dispatch({grads, weights, count, gradn::UPDATE, max_norm, lr, norm, static_cast<double *>(workspace),
                            (cudaStream_t)stream}, total);
}

}  // extern "C"
