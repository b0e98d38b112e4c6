// grad_norm.cu -- the global norm of a network's gradients, clipping by it, and
// the clipped update of Algorithm 1, over lists of tensors.
//
// Two kernels: the first sums the squares, a partial sum per block; every block
// of the second adds the partial sums up again (a few kilobytes from L2, in the
// same order everywhere) and then scales or updates its share.  The tensors'
// addresses and lengths travel as kernel arguments, so a call leaves nothing
// on the device but the partial sums in the caller's workspace.
//
// The tensors are cut into chunks, and a block takes shares of consecutive ones: the host
// tells it the first one's tensor, from there it walks on.  (A search for each
// chunk's tensor through the arguments cost 331 small tensors 11 us of a
// kernel's time.)
//
// Bound by memory: the gradients are read by the first kernel and again by the
// second, which takes the blocks' shares in the opposite order so that what the L2
// still holds is read first.  Norm and clipping of 250 M bf16 values: 248 us, 1.5 GB at
// 6.1 TB/s (the squares 5.5 TB/s, the step 6.0); norm and update of 14 M fp32: 39.8 us,
// of 41 k in one kernel 6.8 us, all latency.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "kernels.cuh"
#include "values.cuh"

namespace cg = cooperative_groups;

namespace minw {
namespace gradn {

constexpr int THREADS = 256;
constexpr int CHUNK = 8 * THREADS;   // values of a chunk: a 16-byte vector of bf16 for each thread
constexpr int SQUARES_PER_SM = 8, STEP_PER_SM = 4;      // resident blocks of the two kernels
constexpr int MAX_BLOCKS = 1216;     // blocks of the first kernel, and so its partial sums, at most
constexpr int MAX_SHARES = 2432;     // shares of a large set: 16 per SM, whole rounds of both kernels
constexpr int CAP_MAX = 864;         // tensors of a launch: with the shares' first tensors, 32.5 KB of the 32764 bytes that
                                     // a launch may pass
constexpr int SMALL_BLOCKS = 8;      // blocks of the cluster that takes a small set
constexpr int SMALL_CHUNKS = 64;     // chunks of a small set at most

enum Op { CLIP = 0, UPDATE = 1 };

struct Entry {
    const void *g;
    void *o;              // clipped gradient, or weights
    uint64_t packed;      // values (42 bits), from bit 48 on the values before the first vector (part of the first chunk),
                          // from bit 56 on types: bit 0 gradients bf16, bit 1 the other tensor bf16, bit 2 both tensors'
                          // vectors are aligned
    uint32_t first;       // first chunk of this tensor
    float limit;

    __host__ __device__ int64_t n() const { return (int64_t)(packed & 0xffffffffffffull); }
    __host__ __device__ int head() const { return (int)(packed >> 48) & 0xff; }
    __host__ __device__ int types() const { return (int)(packed >> 56); }
};

template <int CAP>
struct List {
    Entry e[CAP];
    uint16_t start[MAX_SHARES];      // tensor of a share's first chunk
    int count, shares, each;         // each: chunks of a share
    uint32_t chunks;
};

// Calls f(entry, i0, i1) for the values of each tensor in a share of the chunks.
template <int CAP, typename F>
__device__ __forceinline__ void in_share(const List<CAP> &l, int s, F f) {
    uint32_t c = (uint32_t)s * l.each;
    const uint32_t c1 = min(c + l.each, l.chunks);
    for (int t = l.start[s]; c < c1; ++t) {
        const Entry &e = l.e[t];
        const uint32_t end = t + 1 < l.count ? l.e[t + 1].first : l.chunks, stop = end < c1 ? end : c1;
        const int64_t i0 = c == e.first ? 0 : e.head() + (int64_t)(c - e.first) * CHUNK;
        const int64_t i1 = stop == end ? e.n() : e.head() + (int64_t)(stop - e.first) * CHUNK;
        f(e, i0, i1);
        c = stop;
    }
}

// ... in all of a block's shares, or backwards.
template <int CAP, typename F>
__device__ __forceinline__ void in_block(const List<CAP> &l, bool back, F f) {
    for (int s = blockIdx.x; s < l.shares; s += gridDim.x) in_share(l, back ? l.shares - 1 - s : s, f);
}

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// A sum with what its additions rounded away (Knuth's two-sum): hi + lo.
struct Sum2 {
    float hi = 0.0f, lo = 0.0f;
    __device__ __forceinline__ void add(float v) {
        const float s = hi + v, b = s - hi;
        lo += (hi - (s - b)) + (v - b);
        hi = s;
    }
};

// Squares of this thread's values among [i0, i1): a few at a time in fp32, those sums compensated.  `bits` gathers the
// bits of the values' magnitudes.
template <typename T>
__device__ __forceinline__ void squares(const T *g, int64_t i0, int64_t i1, int head, Sum2 &sum, uint32_t &bits) {
    constexpr int V = 16 / sizeof(T), U = 4;
    constexpr uint32_t MAGNITUDE = sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu;
    const int64_t v0 = i0 == 0 ? head : i0, h1 = v0 < i1 ? v0 : i1;      // first aligned value
    const int64_t nv = (i1 - h1) / V, tail = h1 + nv * V;
    const T *p = g + h1;
    for (int64_t k = threadIdx.x; k < nv; k += U * THREADS) {
        Vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k + u * THREADS < nv) v[u].load(p + (k + u * THREADS) * V);
            else
                for (int w = 0; w < Vec<T, V>::WORDS; ++w) v[u].w[w] = 0;
        }
        Pair s = pair(0.0f, 0.0f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int w = 0; w < Vec<T, V>::WORDS; ++w) bits |= v[u].w[w] & MAGNITUDE;
#pragma unroll
            for (int i = 0; i < V / 2; ++i) s = fma2(v[u].get2(i), v[u].get2(i), s);
        }
        const float2 h = halves(s);
        sum.add(h.x + h.y);
    }
    // the values before the first vector and after the last
    for (int64_t i = i0 + threadIdx.x; i < i1; i += THREADS) {
        if (i >= h1 && i < tail) {
            i += (tail - i - 1) / THREADS * THREADS;
            continue;
        }
        Vec<T, 1> v;
        v.load(g + i);
        bits |= v.w[0] & MAGNITUDE;
        sum.add(v.get(0) * v.get(0));
    }
}

template <typename T>
__device__ __forceinline__ double squares64(const T *g, int64_t i0, int64_t i1) {
    double d = 0.0;
    for (int64_t i = i0 + threadIdx.x; i < i1; i += THREADS) {
        Vec<T, 1> v;
        v.load(g + i);
        d = fma((double)v.get(0), (double)v.get(0), d);
    }
    return d;
}

// Sum of squares of a block's shares (the first thread's value counts).
template <int CAP>
__device__ __forceinline__ double block_squares(const List<CAP> &l) {
    __shared__ float2 red[THREADS / 32];
    __shared__ double red64[THREADS / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Sum2 sum;
    uint32_t bits = 0;
    in_block(l, false, [&](const Entry &e, int64_t i0, int64_t i1) {
        if (e.types() & 1) squares(static_cast<const uint16_t *>(e.g), i0, i1, e.head(), sum, bits);
        else squares(static_cast<const float *>(e.g), i0, i1, e.head(), sum, bits);
    });
    // Squares round to multiples of 2^-149 and overflow at 2^128: where a thread's sum is so small that the former may
    // count (1e5 such roundings are 2^-30 of 1e-31), or near the latter, the block sums its shares again in fp64.
    const bool odd = !(sum.hi >= 1e-31f && sum.hi <= 1e35f) && bits != 0u;
    if (__syncthreads_or(odd)) {
        double d = 0.0;
        in_block(l, false, [&](const Entry &e, int64_t i0, int64_t i1) {
            d += (e.types() & 1) ? squares64(static_cast<const uint16_t *>(e.g), i0, i1)
                               : squares64(static_cast<const float *>(e.g), i0, i1);
        });
        d = warp_sum64(d);
        if (lane == 0) red64[warp] = d;
        __syncthreads();
        if (threadIdx.x == 0)
            for (int k = 1; k < THREADS / 32; ++k) d += red64[k];
        return d;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float hi = __shfl_xor_sync(0xffffffffu, sum.hi, d), lo = __shfl_xor_sync(0xffffffffu, sum.lo, d);
        sum.add(hi);
        sum.lo += lo;
    }
    if (lane == 0) red[warp] = make_float2(sum.hi, sum.lo);
    __syncthreads();
    if (threadIdx.x == 0)
        for (int k = 1; k < THREADS / 32; ++k) {
            sum.add(red[k].x);
            sum.lo += red[k].y;
        }
    return (double)sum.hi + (double)sum.lo;
}

template <int CAP>
__global__ void __launch_bounds__(THREADS, SQUARES_PER_SM) squares_kernel(const __grid_constant__ List<CAP> l, double *part) {
    pdl_trigger();
    pdl_wait();
    const double s = block_squares(l);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// sqrt(s) as an fp32 number, by fp32 instructions (every thread needs it, and fp64 ones take 16 clocks a warp and SM: the
// square root and a quotient in fp64 held the blocks for 8 us): the root of s / 4^e, between 1 and 2, times 2^e.
__device__ __forceinline__ float root(double s) {
    const int64_t bits = __double_as_longlong(s);
    const int ex = (int)(bits >> 52) & 0x7ff;
    if (ex == 0x7ff) return (float)s;                            // infinity, NaN
    if (ex == 0) return 0.0f;                                    // below 2^-1022
    const int e = (ex - 1023) >> 1;
    return ldexpf(sqrtf((float)__longlong_as_double(bits - ((int64_t)(2 * e) << 52))), e);
}

// The norm from the partial sums, by every block alike: a warp adds them up in fp64.
__device__ __forceinline__ float norm_of(const double *part, int parts, double *sum) {
    if (threadIdx.x < 32) {
        double s = 0.0;
#pragma unroll 8
        for (int k = threadIdx.x; k < parts; k += 32) s += part[k];
        s = warp_sum64(s);
        if (threadIdx.x == 0) *sum = s;
    }
    __syncthreads();
    return root(*sum);
}

__global__ void __launch_bounds__(THREADS) norm_kernel(const double *part, int parts, float *norm) {
    pdl_trigger();
    pdl_wait();
    __shared__ double sum;
    const float n = norm_of(part, parts, &sum);
    if (threadIdx.x == 0) *norm = n;
}

template <int OP>
__device__ __forceinline__ float step(float g, float w, float k, float lr, float limit) {
    if (OP == CLIP) return k * g;
    const float v = fmaf(-lr, k * g, w);
    return v > limit ? limit : v < -limit ? -limit : v;
}

// Vectors where both tensors' begin together, else value by value (14 M fp32 in 33 tensors, gradients in one buffer and
// weights of their own allocation: the update 81 us for 40).
template <int OP, typename TG, typename TO>
__device__ __forceinline__ void steps(const Entry &e, int64_t i0, int64_t i1, float k, float lr) {
    constexpr int V = sizeof(TG) == 2 && sizeof(TO) == 2 ? 8 : 4, U = OP == UPDATE ? 2 : 4;
    const TG *g = static_cast<const TG *>(e.g);
    TO *o = static_cast<TO *>(e.o);
    const int64_t v0 = i0 == 0 ? e.head() : i0, h1 = v0 < i1 ? v0 : i1;
    const int64_t nv = (e.types() & 4) ? (i1 - h1) / V : 0, tail = h1 + nv * V;
    for (int64_t j = threadIdx.x; j < nv; j += U * THREADS) {
        Vec<TG, V> vg[U];
        Vec<TO, V> vo[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u * THREADS < nv) {
                vg[u].load(g + h1 + (j + u * THREADS) * V);
                if (OP == UPDATE) vo[u].load(o + h1 + (j + u * THREADS) * V);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j + u * THREADS >= nv) break;
            float r[V];
#pragma unroll
            for (int i = 0; i < V; ++i) r[i] = step<OP>(vg[u].get(i), OP == UPDATE ? vo[u].get(i) : 0.0f, k, lr, e.limit);
            vo[u].set(r);
            vo[u].store(o + h1 + (j + u * THREADS) * V);
        }
    }
    for (int64_t i = i0 + threadIdx.x; i < i1; i += THREADS) {
        if (i >= h1 && i < tail) {
            i += (tail - i - 1) / THREADS * THREADS;
            continue;
        }
        Vec<TG, 1> vg;
        Vec<TO, 1> vo;
        vg.load(g + i);
        if (OP == UPDATE) vo.load(o + i);
        const float r = step<OP>(vg.get(0), OP == UPDATE ? vo.get(0) : 0.0f, k, lr, e.limit);
        vo.set(&r);
        vo.store(o + i);
    }
}

// A block's shares clipped or updated by the norm n.
template <int OP, int CAP>
__device__ __forceinline__ void block_steps(const List<CAP> &l, float n, float max_norm, float lr, float *norm) {
    if (norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
    const bool finite = n <= 3.402823466e38f;                     // false for NaN
    if (OP == UPDATE && !finite) return;
    const float k = finite && n > max_norm ? max_norm / n : 1.0f;
    in_block(l, true, [&](const Entry &e, int64_t i0, int64_t i1) {
        if (OP == CLIP) {
            if (k == 1.0f && e.o == e.g) return;
            if (e.types() & 1) steps<OP, uint16_t, uint16_t>(e, i0, i1, k, lr);
            else steps<OP, float, float>(e, i0, i1, k, lr);
        } else if (e.types() & 2) {
            if (e.types() & 1) steps<OP, uint16_t, uint16_t>(e, i0, i1, k, lr);
            else steps<OP, float, uint16_t>(e, i0, i1, k, lr);
        } else {
            if (e.types() & 1) steps<OP, uint16_t, float>(e, i0, i1, k, lr);
            else steps<OP, float, float>(e, i0, i1, k, lr);
        }
    });
}

template <int OP, int CAP>
__global__ void __launch_bounds__(THREADS, STEP_PER_SM) step_kernel(const __grid_constant__ List<CAP> l, const double *part,
                                                       int parts, float max_norm, float lr, float *norm) {
    pdl_trigger();
    pdl_wait();
    __shared__ double sum;
    block_steps<OP>(l, norm_of(part, parts, &sum), max_norm, lr, norm);
}

// A small set in one kernel: the blocks of one cluster, which read each other's sums.
template <int OP, int CAP>
__global__ void __launch_bounds__(THREADS, STEP_PER_SM) small_kernel(const __grid_constant__ List<CAP> l, float max_norm,
                                                                     float lr, float *norm) {
    pdl_trigger();
    pdl_wait();
    __shared__ double own, all, sums[SMALL_BLOCKS];
    cg::cluster_group cluster = cg::this_cluster();
    const double s = block_squares(l);
    if (threadIdx.x == 0) own = s;
    cluster.sync();
    if (threadIdx.x < gridDim.x) sums[threadIdx.x] = *cluster.map_shared_rank(&own, threadIdx.x);
    __syncthreads();
    cluster_done_reading();
    if (threadIdx.x == 0) {
        double n = sums[0];
        for (int k = 1; k < (int)gridDim.x; ++k) n += sums[k];
        all = n;
    }
    __syncthreads();
    block_steps<OP>(l, root(all), max_norm, lr, norm);
    cluster_leave();
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
        if ((reinterpret_cast<uintptr_t>(l[t].data) & (size_of(l[t].type) - 1)) != 0) return false;
    }
    return true;
}

// Fills one launch's list from tensor t on; returns the next launch's first tensor.
template <int CAP>
static int fill(List<CAP> &l, const minw_tensor *g, const minw_tensor *o, int t, int count) {
    l.count = 0;
    l.chunks = 0;
    for (; t < count && l.count < CAP; ++t) {
        if (g[t].n == 0) continue;
        const int gs = size_of(g[t].type), os = o ? size_of(o[t].type) : 16;
        Entry &e = l.e[l.count];
        e.g = g[t].data;
        e.o = o ? o[t].data : nullptr;
        e.limit = o ? o[t].limit : 0.0f;
        // the head ends where the gradient's 16-byte vectors begin; the other tensor's have to begin there too
        const uint32_t head = (uint32_t)(-reinterpret_cast<uintptr_t>(e.g) & 15) >> (gs == 2 ? 1 : 2);
        const uint32_t vector = gs == 2 && os == 2 ? 16 : 4 * (uint32_t)os;      // its bytes of a vector
        const bool vec = o && ((reinterpret_cast<uintptr_t>(e.o) + head * (uint32_t)os) & (vector - 1)) == 0;
        const uint64_t types = (g[t].type == MINW_BF16 ? 1 : 0) | (o && o[t].type == MINW_BF16 ? 2 : 0) | (vec ? 4 : 0);
        e.packed = (uint64_t)g[t].n | (uint64_t)head << 48 | types << 56;
        const int64_t chunks = g[t].n > head ? (g[t].n - head + CHUNK - 1) / CHUNK : 1;
        e.first = l.chunks;
        l.chunks += (uint32_t)chunks;
        ++l.count;
    }
    while (t < count && g[t].n == 0) ++t;                             // no launch for empty tensors alone
    // a share is a chunk, a block's part of a small set, or a MAX_SHARES-th of a large one, so that the blocks move over
    // it side by side (one long share for each block: the clipping of 250 M bf16 values took 294 us for 255)
    const uint32_t most = l.chunks <= (uint32_t)SMALL_CHUNKS ? SMALL_BLOCKS : MAX_SHARES;
    l.each = (int)((l.chunks + most - 1) / most);
    l.shares = l.chunks ? (int)((l.chunks + l.each - 1) / l.each) : 0;
    for (int k = 0, b = 0; k < l.count; ++k) {
        // the shares whose first chunk comes before the next tensor's
        const uint32_t end = k + 1 < l.count ? l.e[k + 1].first : l.chunks;
        for (; (uint32_t)b * l.each < end; ++b) l.start[b] = (uint16_t)k;
    }
    return t;
}

static int blocks_of(int shares, int per_sm) {
    const int sms = num_sms() > 0 ? num_sms() : 152, cap = sms * per_sm < MAX_BLOCKS ? sms * per_sm : MAX_BLOCKS;
    return shares < cap ? shares : cap;
}

struct Call {
    const minw_tensor *g, *o;
    int count, op;               // op -1: the norm alone
    float max_norm, lr;
    float *norm;
    double *part;
    cudaStream_t s;
};

template <typename... A>
static cudaError_t launch_small(void (*kern)(A...), int blocks, cudaStream_t s, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)blocks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <int CAP>
static minw_status run(const Call &c) {
    List<CAP> l;                      // at most 32 KB
    int parts = 0, launches = 0;
    for (int t = 0; t < c.count;) {
        t = fill(l, c.g, c.o, t, c.count);
        if (l.chunks == 0) continue;
        if constexpr (CAP <= 128)                      // a longer list has more chunks
            if (launches == 0 && t >= c.count && c.op >= 0 && l.chunks <= (uint32_t)SMALL_CHUNKS)
                return launch_small(c.op == CLIP ? small_kernel<CLIP, CAP> : small_kernel<UPDATE, CAP>, l.shares, c.s, l,
                                    c.max_norm, c.lr, c.norm) == cudaSuccess
                           ? launch_status()
                           : launch_failed();
        const int blocks = blocks_of(l.shares, SQUARES_PER_SM);
        if (launch_pdl_stream(false, squares_kernel<CAP>, dim3((unsigned)blocks), dim3(THREADS), 0, c.s, l,
                              c.part + parts) != cudaSuccess)
            return launch_failed();
        parts += blocks;
        ++launches;
    }
    if (c.op < 0 || parts == 0) {
        if (launch_pdl_stream(false, norm_kernel, dim3(1), dim3(THREADS), 0, c.s, (const double *)c.part, parts,
                              c.norm) != cudaSuccess)
            return launch_failed();
        return launch_status();
    }
    float *norm = c.norm;
    for (int t = 0; t < c.count;) {
        if (launches > 1) t = fill(l, c.g, c.o, t, c.count);
        else t = c.count;                                                    // the list is still the one launch's
        if (l.chunks == 0) continue;
        if (launch_pdl_stream(false, c.op == CLIP ? step_kernel<CLIP, CAP> : step_kernel<UPDATE, CAP>,
                              dim3((unsigned)blocks_of(l.shares, STEP_PER_SM)), dim3(THREADS), 0, c.s, l,
                              (const double *)c.part, parts, c.max_norm, c.lr, norm) != cudaSuccess)
            return launch_failed();
        norm = nullptr;
    }
    return launch_status();
}

static minw_status check(const minw_tensor *g, const minw_tensor *o, int count, const float *norm, const void *ws,
                         size_t ws_bytes, bool same_types) {
    if (count < 0 || (count > 0 && !g) || !norm || !ws) return MINW_EINVAL;
    if (!aligned16(ws) || ws_bytes < minw_grad_workspace_bytes(count)) return MINW_EINVAL;
    if (reinterpret_cast<uintptr_t>(norm) % 4 != 0) return MINW_EINVAL;
    if (!valid_list(g, count) || (o && !valid_list(o, count))) return MINW_EINVAL;
    int64_t total = 0;
    for (int t = 0; t < count; ++t) {
        if (o && (o[t].n != g[t].n || (same_types && o[t].type != g[t].type))) return MINW_EINVAL;
        if (g[t].n >= (1ll << 42) || (total += g[t].n) >= (1ll << 42)) return MINW_EUNSUPPORTED;
    }
    return MINW_OK;
}

// The list's capacity decides how many bytes of arguments a launch carries.
static minw_status dispatch(const Call &c) {
    return c.count <= 16 ? run<16>(c) : c.count <= 128 ? run<128>(c) : c.count <= 384 ? run<384>(c) : run<CAP_MAX>(c);
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
    const minw_status st = gradn::check(grads, nullptr, count, norm, workspace, workspace_bytes, false);
    if (st != MINW_OK) return st;
    return gradn::dispatch({grads, nullptr, count, -1, 0.0f, 0.0f, norm, static_cast<double *>(workspace),
                            (cudaStream_t)stream});
}

minw_status minw_grad_clip(const minw_tensor *grads, const minw_tensor *out, int32_t count, float max_norm, float *norm,
                           void *workspace, size_t workspace_bytes, void *stream) {
    if (count > 0 && !out) return MINW_EINVAL;
    if (!(max_norm > 0.0f && isfinite(max_norm))) return MINW_EINVAL;
    const minw_status st = gradn::check(grads, out, count, norm, workspace, workspace_bytes, true);
    if (st != MINW_OK) return st;
    return gradn::dispatch({grads, out, count, gradn::CLIP, max_norm, 0.0f, norm, static_cast<double *>(workspace),
                            (cudaStream_t)stream});
}

minw_status minw_sgd_clip_norm(const minw_tensor *weights, const minw_tensor *grads, int32_t count, float max_norm,
                               float lr, float *norm, void *workspace, size_t workspace_bytes, void *stream) {
    if (count > 0 && !weights) return MINW_EINVAL;
    if (!(max_norm > 0.0f && isfinite(max_norm)) || !isfinite(lr)) return MINW_EINVAL;
    const minw_status st = gradn::check(grads, weights, count, norm, workspace, workspace_bytes, false);
    if (st != MINW_OK) return st;
    for (int t = 0; t < count; ++t)
        if (!(weights[t].limit >= 0.0f)) return MINW_EINVAL;
    return gradn::dispatch({grads, weights, count, gradn::UPDATE, max_norm, lr, norm, static_cast<double *>(workspace),
                            (cudaStream_t)stream});
}

}  // extern "C"
