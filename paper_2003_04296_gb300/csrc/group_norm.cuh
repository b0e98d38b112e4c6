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
    // one pass
    int butterfly;                 // lanes and the lanes of a group are powers of two within a warp
    int rows, groups, per;         // pixel rows of a block, groups of a slab, entries (a thread's share of a group) of a group
    float inv_total;               // 1 / (P Cg)
    int seg;                       // backward: threads that sum a channel's rows
    Div by_L, by_rows, by_per, by_chunks, by_slabs, by_channels;
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
// One pass: an image's slab of whole groups (L lanes of V channels) stays in
// the registers of a block, or of a cluster of blocks that split its pixels;
// x (and dy) are read once.
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

// Pixel chunks per image of the streaming kernels: about eight blocks per SM over all images, at least 64 pixels each.
inline int chunks_of(int B, int64_t P) {
    int64_t k = (8 * 152 + B - 1) / B;
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
    l.part = take((size_t)B * chunks_of(B, P) * C);
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

// Lanes and slabs of the streaming kernels for V channels a lane.
inline void lanes(Args &a, int V) {
    const int lanes = a.C / V;
    a.slabs = (lanes + THREADS - 1) / THREADS;
    a.L = (lanes + a.slabs - 1) / a.slabs;
}

// The one-pass plan: slabs of whole groups, at least 128 bytes of a row wide where one fits (64, then 32 where not), the
// narrowest such, so that the blocks are many and their clusters small; clusters of at most 16 blocks of
// THREADS / L rows of NV pixels.
struct Plan {
    int V, GPT, NV;
};
inline bool one_pass(Args &a, Plan &pl, int bytes, int V0, bool backward) {
    pl.V = V0 == 8 && a.Cg % 2 != 0 ? 4 : V0;
    pl.GPT = a.Cg % pl.V == 0 ? 1 : pl.V == 8 ? (a.Cg % 4 == 0 ? 2 : 4) : a.Cg % 2 == 0 ? 2 : pl.V;
    for (int width = 128; width >= 32; width /= 2)
        for (int k = 1; k <= a.G && k <= MAX_SLAB_GROUPS; ++k) {
            const int channels = k * a.Cg;
            if (a.G % k != 0 || channels % pl.V != 0 || (channels * bytes < width && k < a.G)) continue;
            const int L = channels / pl.V;
            if (L > THREADS) break;
            const int rows = THREADS / L;
            // the backward holds two tensors, so never more than 8 vectors of each
            pl.NV = pl.V == 1 ? 32 : backward || a.P <= 64 * rows ? 8 : 16;
            const int64_t cap = (int64_t)rows * pl.NV, cluster = (a.P + cap - 1) / cap;
            if (cluster > 16 || (backward && cluster > 1 && rows < 2)) break;     // a cluster's totals go behind the block's sums
            a.per = a.Cg / (pl.V / pl.GPT);
            a.butterfly = L <= 32 && (L & (L - 1)) == 0 && (a.per == 1 || (pl.GPT == 1 && (a.per & (a.per - 1)) == 0));
            a.rows = rows;
            a.groups = k;
            a.L = L;
            a.slabs = a.G / k;
            a.inv_total = (float)(1.0 / ((double)a.P * a.Cg));
            a.seg = channels >= THREADS ? 1 : THREADS / channels < rows ? THREADS / channels : rows;
            a.by_channels = Div((uint32_t)channels);
            a.by_L = Div(L);
            a.by_rows = Div(rows);
            a.by_per = Div(a.per);
            a.by_chunks = Div((uint32_t)cluster);
            a.by_slabs = Div((uint32_t)a.slabs);
            a.chunks = (int)cluster;
            a.ppc = (int)((a.P + cluster - 1) / cluster);
            return true;
        }
    return false;
}

inline cudaError_t launch_cluster(void (*kern)(Args), int64_t blocks, cudaStream_t s, const Args &a) {
    if (a.chunks > 8 && !allow_large_clusters(reinterpret_cast<const void *>(kern))) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.chunks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

}  // namespace gn
}  // namespace minw
