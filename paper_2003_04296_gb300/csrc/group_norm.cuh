// group_norm.cuh -- what the forward and the backward of the group norm with an
// activation on channels-last rows share.
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
#pragma once

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
    int wide_affine;               // both given, on 16-byte boundaries
    const float *mean_in, *rstd_in;
    float *mean, *rstd;            // forward: saved statistics (nullable)
    float2 *part;                  // per image, cluster of chunks and group, or chunk and channel: (mean, M2); the backward's
                                   // per image, chunk and channel (sum dz, sum dz xh)
    float2 *stat;                  // streaming: per image and group (mean, rstd), or (s1, s2)
    float2 *chan;                  // backward: per image and channel (sum dz, sum dz xh)
    float *dgamma, *dbeta;         // nullable
    int B, P, C, G, Cg, act;
    float eps;
    int chunks, ppc;               // pixel chunks per image, pixels per chunk
    int L, slabs;                  // lanes (V channels each) of a slab, slabs of a row
    // slabs of whole groups
    int butterfly;                 // forward: lanes and the lanes of a group are powers of two within a warp
    int rows, groups, per;         // pixel rows of a block, groups of a slab, entries (a thread's share of a group) of a group
                                   // (forward)
    float inv_total;               // 1 / (P Cg)
    int seg;                       // backward: threads that sum a channel's rows
    Div by_L, by_rows, by_per, by_Cg, by_chunks, by_slabs, by_channels;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// gamma and beta of channels c .. c + V - 1.
template <int V>
__device__ __forceinline__ void load_affine(const Args &a, int c, float *ga, float *be) {
    if (V >= 4 && a.wide_affine) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 g = *reinterpret_cast<const float4 *>(a.gamma + c + i), b = *reinterpret_cast<const float4 *>(a.beta + c + i);
            ga[i] = g.x; ga[i + 1] = g.y; ga[i + 2] = g.z; ga[i + 3] = g.w;
            be[i] = b.x; be[i + 1] = b.y; be[i + 2] = b.z; be[i + 3] = b.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        ga[i] = a.gamma ? a.gamma[c + i] : 1.0f;
        be[i] = a.beta ? a.beta[c + i] : 0.0f;
    }
}

// U pixels, or one, into the means m and M2 q of the i before them.
template <typename T, int V, int U>
__device__ __forceinline__ void merge_pixels(const Vec<T, V> *v, int i, Pair *m, Pair *q) {
    const float share = __fdividef((float)U, (float)(i + U)), cross = (float)i * share;
    const Pair inv = pair(1.0f / U, 1.0f / U), sh = pair(share, share), cr = pair(cross, cross), minus = pair(-1.0f, -1.0f);
#pragma unroll
    for (int k = 0; k < (V + 1) / 2; ++k) {
        Pair s = v[0].get2(k);
#pragma unroll
        for (int u = 1; u < U; ++u) s = add2(s, v[u].get2(k));
        s = mul2(s, inv);
        const Pair ns = mul2(s, minus);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Pair d = add2(v[u].get2(k), ns);
            q[k] = fma2(d, d, q[k]);
        }
        const Pair d = fma2(m[k], minus, s);
        m[k] = fma2(d, sh, m[k]);
        q[k] = fma2(mul2(d, d), cr, q[k]);
    }
}
template <typename T, int V>
__device__ __forceinline__ void merge_pixel(const Vec<T, V> &v, int i, Pair *m, Pair *q) {
    const float share = __fdividef(1.0f, (float)(i + 1)), cross = (float)i * share;
    const Pair sh = pair(share, share), cr = pair(cross, cross), minus = pair(-1.0f, -1.0f);
#pragma unroll
    for (int k = 0; k < (V + 1) / 2; ++k) {
        const Pair d = fma2(m[k], minus, v.get2(k));
        m[k] = fma2(d, sh, m[k]);
        q[k] = fma2(mul2(d, d), cr, q[k]);
    }
}

// Statistics of a thread's n pixels, `step` values apart, of V channels: means and M2 of each channel, in pairs.  U pixels
// at a time: their mean and M2 by themselves, merged into the channel's.
template <typename T, int V, int U>
__device__ __forceinline__ void channel_stats(const T *x, int64_t step, int n, Pair *m, Pair *q) {
    constexpr int NP = (V + 1) / 2;
#pragma unroll
    for (int k = 0; k < NP; ++k) m[k] = q[k] = pair(0.0f, 0.0f);
    int i = 0;
    for (; i + U <= n; i += U, x += U * step) {
        Vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u].load(x + u * step);
        merge_pixels<T, V, U>(v, i, m, q);
    }
    if (i == n) return;
    // the last few: their loads together, then one by one
    Vec<T, V> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (i + u < n) v[u].load(x + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (i + u >= n) break;
        merge_pixel<T, V>(v[u], i + u, m, q);
    }
}

// The same through a ring of asynchronous copies: eight pixels of a thread in flight without a register of them, and the
// last ones, from first() on, stay there.  Each thread reads its own copies, so that the ring needs no barrier.
constexpr int RING_PIXELS = 8;
template <typename T, int V>
struct Ring {
    static constexpr int U = 4, BYTES = Vec<T, V>::BYTES, SIZE = RING_PIXELS * THREADS * BYTES;
    static_assert(RING_PIXELS == 2 * U, "two fetches in flight");
    uint8_t *own;
    __device__ __forceinline__ explicit Ring(uint8_t *shared) : own(shared + threadIdx.x * BYTES) {}
    static __device__ __forceinline__ int first(int n) { return max((n + U - 1) / U * U - RING_PIXELS, 0); }
    __device__ __forceinline__ uint8_t *slot(int i) const { return own + (i & (RING_PIXELS - 1)) * (THREADS * BYTES); }
    __device__ __forceinline__ Vec<T, V> read(int i) const {
        Vec<T, V> v;
        v.load(reinterpret_cast<const T *>(slot(i)));
        return v;
    }
    __device__ __forceinline__ void stats(const T *x, int64_t step, int n, Pair *m, Pair *q) const {
        auto fetch = [&](int i0) {                              // pixels i0 .. i0 + U - 1, those that there are
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u < n) copy_async<BYTES>(slot(i0 + u), x + u * step);
            x += U * step;
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll
        for (int k = 0; k < (V + 1) / 2; ++k) m[k] = q[k] = pair(0.0f, 0.0f);
        fetch(0);
        fetch(U);
        int i = 0;
        for (; i + U <= n; i += U) {
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            Vec<T, V> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = read(i + u);
            merge_pixels<T, V, U>(v, i, m, q);
            fetch(i + RING_PIXELS);
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        for (; i < n; ++i) merge_pixel<T, V>(read(i), i, m, q);
    }
};

// f(u) for a thread's n pixels, U at a time, after load(u) for all of those; once() when the first are on their way.
template <int U, typename L, typename O, typename F>
__device__ __forceinline__ void batches(int n, L load, O once, F f) {
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < n) load(u);
    once();
    int i = 0;
    for (; i + U <= n; i += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) f(u);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + U + u < n) load(u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (i + u < n) f(u);
}

// y = act((x - mean) a + b) on a pixel.
template <typename T, typename TY, int V, int ACT>
__device__ __forceinline__ void apply_pixel(const Vec<T, V> &v, TY *y, const Pair *nm, const Pair *a, const Pair *b) {
    constexpr int NP = (V + 1) / 2;
    float z[2 * NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        const float2 h = halves(fma2(add2(v.get2(k), nm[k]), a[k], b[k]));
        z[2 * k] = act_value<ACT>(h.x);
        z[2 * k + 1] = act_value<ACT>(h.y);
    }
    Vec<TY, V> o;
    o.set(z);
    o.store(y);
}

// The same on a thread's n pixels: minus the means, a = rstd gamma and b = beta in pairs.  From the last pixel to the
// first: what the sums read last is what L2 still holds (2 x 252003 x 96 of 160: 68.4 us for 69.8 in the sums' order,
// 64 x 112 x 112 x 64: 55.7 for 56.9).
template <typename T, typename TY, int V, int U, int ACT, typename K>
__device__ __forceinline__ void apply_pixels(const T *x, int64_t xstep, TY *y, int64_t ystep, int first, int n, K kept,
                                             const Pair *nm, const Pair *a, const Pair *b) {
    Vec<T, V> v[U];
    if (V > 1) {
        x += (first - 1) * xstep;
        y += (n - 1) * ystep;
        xstep = -xstep;
        ystep = -ystep;
    }
    batches<U>(
        first,
        [&](int u) {
            v[u].load(x);
            x += xstep;
        },
        [&] {
#pragma unroll 4
            for (int i = n - 1; i >= first; --i, y += ystep) apply_pixel<T, TY, V, ACT>(kept(i), y, nm, a, b);
        },
        [&](int u) {
            apply_pixel<T, TY, V, ACT>(v[u], y, nm, a, b);
            y += ystep;
        });
}

// Where a block of the streaming kernels works: image, chunk of its pixels, slab of its channels.
struct Place {
    int b, chunk, slab, p0, p1, rows, row, lane, c, n;
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
    w.lane = (int)threadIdx.x % a.L;
    w.c = (w.slab * a.L + w.lane) * V;
    const bool some = w.row < w.rows && w.c < a.C && w.p0 + w.row < w.p1;
    w.n = some ? (w.p1 - w.p0 - w.row - 1) / w.rows + 1 : 0;
    return w;
}

// ---------------------------------------------------------------------------
// One kernel: a block, or a cluster of blocks that split the pixels, takes an
// image's slab of whole groups (L lanes of V channels).  A slab stays in shared
// memory where there are no more slabs than the SMs can hold at a time, in a
// block's registers where there are and it fits; of larger ones, what has left
// the block's ring is read again, from L2, once their sums are known.
// ---------------------------------------------------------------------------

constexpr int MAX_SLAB_GROUPS = 256;

struct Tile {
    int b, slab, rank, p0, p1, lane, row, rows, c, n;      // n: pixels of this thread
};
template <int V>
__device__ __forceinline__ Tile tile(const Args &a) {
    Tile w;
    const int bs = a.by_chunks.div((int)blockIdx.x);
    w.rank = (int)blockIdx.x - bs * a.chunks;
    w.b = a.by_slabs.div(bs);
    w.slab = bs - w.b * a.slabs;
    w.p0 = min(a.P, w.rank * a.ppc);
    w.p1 = min(a.P, w.p0 + a.ppc);
    w.row = a.by_L.div((int)threadIdx.x);
    w.lane = (int)threadIdx.x - w.row * a.L;
    w.rows = a.rows;
    w.c = (w.slab * a.L + w.lane) * V;
    w.n = w.row < w.rows && w.p0 + w.row < w.p1 ? a.by_rows.div(w.p1 - w.p0 - w.row - 1) + 1 : 0;
    return w;
}

// Halves 2 k and 2 k + 1 of V values (the second 0 for a single one).
template <int V>
__device__ __forceinline__ Pair pick(const float *f, int k) {
    return pair(f[2 * k], V > 1 ? f[2 * k + 1] : 0.0f);
}
// The same from one value per group of W channels, negated or not.
template <int V, int W>
__device__ __forceinline__ Pair pick_group(const float *f, int k, float sign = 1.0f) {
    return pair(sign * f[2 * k / W], V > 1 ? sign * f[(2 * k + 1) / W] : 0.0f);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

using namespace minw_host;

inline size_t al256(size_t v) { return (v + 255) & ~(size_t)255; }

// Resident blocks of the streaming kernels (half of them in the backward), and the chunks that a cluster merges.
constexpr int STREAM_BLOCKS = 4 * 152, STREAM_CLUSTER = 4;

// Pixel chunks per image for B images of so many slabs, at least 64 pixels each.
inline int chunks_of(int blocks, int B, int slabs, int64_t P) {
    int64_t k = blocks / ((int64_t)B * slabs);
    if (k > (P + 63) / 64) k = (P + 63) / 64;
    return (int)(k < 1 ? 1 : k);
}

struct Layout {
    size_t part, stat, chan, total;
};
inline Layout layout(int B, int64_t P, int C, int G, bool backward) {
    Layout l;
    size_t off = 0;
    auto take = [&](size_t n) { const size_t r = off; off += al256(n * sizeof(float2)); return r; };
    const int64_t chunks = B * ((P + 63) / 64), most = B > STREAM_BLOCKS ? B : STREAM_BLOCKS;       // of all images
    l.part = take((size_t)(chunks < most ? chunks : most) * C);
    l.stat = take((size_t)B * G);
    l.chan = backward ? take((size_t)B * C) : off;
    l.total = off;
    return l;
}

inline bool valid_type(int t) { return t == MINW_F32 || t == MINW_BF16; }
inline int bytes_of(int t) { return t == MINW_BF16 ? 2 : 4; }

// Whether a tensor's rows start on multiples of V values (at most 16 bytes of them).
inline bool fits(const void *p, int64_t ld, int type, int V) {
    const int bytes = bytes_of(type) * V > 16 ? 16 : bytes_of(type) * V;
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * bytes_of(type) % bytes == 0;
}

// An output at an input's address replaces it value by value.
inline bool in_place_ok(const void *in, int in_type, int64_t in_ld, const void *out, int out_type, int64_t out_ld) {
    return in == nullptr || in != out || (in_type == out_type && in_ld == out_ld);
}

inline cudaError_t launch(void (*kern)(Args), int64_t blocks, cudaStream_t s, const Args &a) {
    return launch_pdl_stream(false, kern, dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
}

// Lanes and slabs, V channels a lane, without regard to groups.
inline void lanes(Args &a, int V) {
    const int all = a.C / V;
    a.slabs = (all + THREADS - 1) / THREADS;
    a.L = (all + a.slabs - 1) / a.slabs;
    a.by_Cg = Div(a.Cg);
}

// The plan for slabs of whole groups: at least 128 bytes of a row wide where one fits (64 where not, or where the wide
// ones are too few to fill the SMs), the narrowest such, so that the blocks are many.  The memory's lines are 128 bytes:
// the backward of 256 x 256 x 256 bf16 takes 32.0 us in slabs of 128 bytes, 40.1 of 64; that of 2 x 64 x 512 4.7 of 64,
// 5.1 of 128.  Whole lines where rows begin on one: 100 x 2000 x 96 fp32 53.6 us, 58.2 without.
enum Way { SHARED, HELD, REREAD, CHUNKS };      // in shared memory, in registers, read twice; images in chunks
struct Plan {
    int V, GPT;
    Way way;
    int smem;                                   // of a block: its vectors
};
constexpr int SHARED_MOST = 100 * 1024;         // (two blocks per SM)
inline bool plan(Args &a, Plan &pl, int bytes, int dy_bytes, int V0) {
    const bool backward = dy_bytes != 0;
    const int sms = num_sms() > 0 ? num_sms() : 152, places = (backward ? 2 : 4) * sms;      // resident blocks
    pl.V = V0 == 8 && a.Cg % 2 != 0 && !backward ? 4 : V0;
    pl.GPT = a.Cg % pl.V == 0 ? 1 : pl.V == 8 ? (a.Cg % 4 == 0 ? 2 : 4) : a.Cg % 2 == 0 ? 2 : pl.V;
    int k = 0, channels = 0, L = 0, rows = 0, cluster = 0;
    // t groups make a slab: whole lines of rows that begin on one, whole rows, or at least `width` bytes
    auto slab = [&](int width, bool lines) {
        for (int t = 1; t <= a.G && t <= MAX_SLAB_GROUPS && t * a.Cg / pl.V <= THREADS; ++t) {
            if (a.G % t != 0 || t * a.Cg % pl.V != 0 || t * a.Cg * bytes < (t == a.G ? 0 : width)) continue;
            if (lines && t != a.G && (t * a.Cg * bytes % 128 != 0 || a.ldx * bytes % 128 != 0)) continue;
            if (lines && t * a.Cg * bytes > 512) break;
            k = t;
            return;
        }
    };
    slab(128, true);
    if (k == 0) slab(128, false);
    const int wide = k;
    if (k == 0 || (int64_t)a.B * (a.G / k) * 8 < places) slab(64, false);
    if (wide != 0 && (int64_t)a.B * (a.G / k) * 8 < sms) k = wide;      // images in chunks: the chunks fill the SMs
    if (k == 0) slab(32, false);
    if (k == 0) return false;
    channels = k * a.Cg;
    L = channels / pl.V;
    rows = THREADS / L;
    const int64_t slabs = (int64_t)a.B * (a.G / k);
    const int cap = rows * (pl.V == 1 ? 32 : 8);
    cluster = 1;
    // Registers hold eight pixels of a thread.  A cluster's registers for more lose to a second reading that a ring
    // spares in part: 200 x 784 x 256 fp32 60.0 us in two readings, 67.6 in clusters of four, the backward 92.6 and 120;
    // at one block 200 x 256 x 256 takes 19.3 us for 21.8, the backward 35.1 for 37.3.
    pl.way = a.P <= cap ? HELD : REREAD;
    pl.smem = 0;
    if (pl.V > 1) {
        auto share = [&](int n) { return (int64_t)((a.P + n - 1) / n + rows - 1) / rows * THREADS * pl.V * (bytes + dy_bytes); };
        // the kernels' own shared memory: sums and statistics, or the channels' sums of the rows
        const int static_bytes = backward ? 8 * THREADS * (pl.V + 1) + 12 * MAX_SLAB_GROUPS
                                          : 8 * (THREADS * pl.GPT + MAX_SLAB_GROUPS) + 16 * MAX_SLAB_GROUPS;
        // clusters of more than two blocks leave up to a tenth of the places empty
        auto resident = [&](int n) {
            const int64_t each = 227 * 1024 / (share(n) + static_bytes + 1024), most = backward ? 2 : 3;
            return share(n) <= SHARED_MOST && slabs * n <= (each < most ? each : most) * sms * (n > 2 ? 9 : 10) / 10;
        };
        // 128 x 784 x 128 bf16: 13.2 us; 14.7 in two readings.  64 x 196 x 256: 5.3 us for 4.8 in registers, 6.4 in two.
        int n = 1;
        while (n <= 8 && !resident(n)) ++n;
        if (n <= 8) {
            // two blocks per SM where a thread keeps four pixels (8 x 1024 x 128: 4.7 us for 5.0)
            while (n <= 4 && slabs * n * 2 <= 2 * sms && a.P >= 8 * n * rows && resident(2 * n)) n *= 2;
            cluster = n;
            pl.way = SHARED;
            pl.smem = (int)share(n);
        }
    }
    if (pl.way == REREAD) {
        // Forward: up to twice as many blocks as fit at a time (160 x 3000 x 128 bf16: 68.6 us; 77.4 with up to as many;
        // 64 x 6000 x 64 loses, 32.3 for 29.6), but not by single values (100 x 400 x 99: 14.1 us, 18.5).  Backward: as many as fit; twice as many where a thread has 16 to 32 pixels
        // then (128 x 3136 x 64: 50.9 us for 54.3) or a third of the places stay empty (100 x 9000 x 64: 117 for 127),
        // and not else (150 x 12544 x 64: 200 us, 239 with twice as many).
        for (cluster = 1; cluster < 8 && slabs * cluster * 2 <= (backward || pl.V == 1 ? 1 : 2) * places; cluster *= 2) {}
        if (backward && cluster < 8 && slabs * cluster <= places && a.P >= 32 * cluster * rows &&
            (a.P < 64 * cluster * rows || slabs * cluster * 10 <= places * 7))
            cluster *= 2;
        // fewer blocks than SMs (2 x 252003 x 96 of 160: 63.7 us, 622 in clusters)
        if (slabs * cluster < sms) pl.way = CHUNKS;
        if (pl.V > 1) pl.smem = RING_PIXELS * THREADS * pl.V * (bytes + dy_bytes);
    }
    // a cluster's totals go behind the block's sums
    if (backward && (pl.way == CHUNKS || (cluster > 1 && rows < 2))) return false;
    if (!backward) {
        // (the backward sums by channels: it has no entries, and its V may be more than two groups of one channel)
        a.per = a.Cg / (pl.V / pl.GPT);
        a.butterfly = L <= 32 && (L & (L - 1)) == 0 && (a.per == 1 || (pl.GPT == 1 && (a.per & (a.per - 1)) == 0));
        a.by_per = Div(a.per);
    }
    a.rows = rows;
    a.groups = k;
    a.L = L;
    a.slabs = a.G / k;
    a.chunks = cluster;
    a.ppc = (a.P + cluster - 1) / cluster;
    a.inv_total = (float)(1.0 / ((double)a.P * a.Cg));
    a.seg = channels >= THREADS ? 1 : THREADS / channels < rows ? THREADS / channels : rows;
    a.by_channels = Div((uint32_t)channels);
    a.by_L = Div(L);
    a.by_rows = Div(rows);
    a.by_Cg = Div(a.Cg);
    a.by_chunks = Div((uint32_t)cluster);
    a.by_slabs = Div((uint32_t)a.slabs);
    return true;
}

// Chunks of images: for the kernels that merge clusters of them (the last chunks may then be empty), or not.
inline bool in_chunks(Args &a, bool clusters, int64_t &blocks) {
    a.chunks = chunks_of(a.dy ? STREAM_BLOCKS / 2 : STREAM_BLOCKS, a.B, a.slabs, a.P);
    a.ppc = (a.P + a.chunks - 1) / a.chunks;
    a.chunks = (a.P + a.ppc - 1) / a.ppc;                           // no chunk without a pixel
    if (clusters) a.chunks = (a.chunks + STREAM_CLUSTER - 1) / STREAM_CLUSTER * STREAM_CLUSTER;
    a.by_chunks = Div((uint32_t)a.chunks);
    blocks = (int64_t)a.B * a.chunks * a.slabs;
    return blocks < (1ll << 31) && (int64_t)a.B * a.G < (1ll << 31);
}

inline cudaError_t launch_cluster(void (*kern)(Args), int64_t blocks, int cluster, int smem, cudaStream_t s, const Args &a) {
    // (48 KB without it, the kernel's own included)
    if (smem > 0 && !allow_shared(reinterpret_cast<const void *>(kern), SHARED_MOST)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

}  // namespace gn
}  // namespace minw
