// adapters.cuh -- what the kernels of low-rank adapters share.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kernels.cuh"
#include "split.cuh"
#include "values.cuh"

namespace cg = cooperative_groups;

namespace minw {
namespace adapters {

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int MAX_RANK = 256;
constexpr int SMALL = 64;                     // rows that need no plan

// ---------------------------------------------------------------------------
// The plan: rows sorted by user, in their order; tiles of at most `most` rows
// ---------------------------------------------------------------------------

struct Tile {
    int id, start, count, pad;               // user (-1: none), place of its first row in the sorted order; pad: one load of 16 bytes
};

struct Plan {
    int *order;                              // [T] the rows, sorted
    int *first;                              // [n + 2] place of each user's first row; n: rows of no user
    int *tiles_n;
    Tile *tiles;
    int *counts;                             // [n + 1][COUNTS] where they exceed shared memory
};

__device__ __forceinline__ int user_of(int id, int n) { return id >= 0 && id < n ? id : n; }

// ---------------------------------------------------------------------------
// Through an adapter
// ---------------------------------------------------------------------------

__device__ __forceinline__ void prefetch(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

struct Args {
    const void *in;                          // [T][D], rows ld_in apart
    const int *ids;
    const void *p1, *p2;                     // [n][r][D], [n][r][E]
    const float *alpha;                      // [n], or null: 1
    const void *base;                        // [T][E], or null: 0
    const float *scale, *shift;              // [E], or null: 1 and 0
    void *out;                               // [T][E]
    float *h;                                // [T][r] by row, or null: in p1^T
    const float *h_in;                       // backward: [T][r] by row ...
    uint16_t *hp, *hh;                       // [3][T][rp] by sorted row, in parts: alpha times the values here, alpha times h_in
    int64_t ld_in, ld_base, ld_out;
    int T, D, E, n, r, rp;                   // rp: r rounded up to 16
    int act, base_bf16, out_bf16;
    int in_vec, p1_vec, p2_vec, base_vec, out_vec;        // whole rows on 16-byte boundaries
    int most;                                // rows of a plan's tile
    int scale_vec;                           // scale and shift on 16-byte boundaries
    int fine;                                // products of parts down to 2^-25
    int split;                               // blocks of a cluster
    Plan plan;
};

template <typename V>
__device__ __forceinline__ void load16(const void *p, int64_t at, int left, float *v) {
    const V *q = static_cast<const V *>(p) + at;
#pragma unroll
    for (int k = 0; k < 16; k += 8) {
        Eight<V> e;
        e.template load<true>(q + k, left - k);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[k + i] = __uint_as_float(sizeof(V) == 4 ? e.w[i % (2 * sizeof(V))] : (i & 1) ? e.w[i >> 1] & 0xffff0000u : e.w[i >> 1] << 16);
    }
}

template <typename V>
__device__ __forceinline__ void store16(void *p, int64_t at, int left, bool vec, const float *v) {
    V *q = static_cast<V *>(p) + at;
    if (vec && left >= 16) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            Vec<V, 8> w;
            w.set(v + 8 * k);
            w.store(q + 8 * k);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < left) {
                Vec<V, 1> w;
                w.set(v + i);
                w.store(q + i);
            }
    }
}

// acc(m) += 32 values along K of MT tiles of 16 rows times those of eight ranks, in parts, the smallest products first.  The tensor
// cores truncate what they add to, so they start these from zero and the sums over K are added here, to nearest: a sum of one
// sign loses no more the longer it gets.
template <int PI, int PP, int MT, typename F>
__device__ __forceinline__ void add_products(const uint32_t (&xp)[MT][2][PI][4], const uint32_t (&pp)[PP][4], F acc) {
    float sum[MT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[m][i] = 0.0f;
#pragma unroll
    for (int l = 2; l >= 0; --l)
#pragma unroll
        for (int q = 0; q <= l; ++q) {
            const int v = l - q;
            if (q >= PI || v >= PP) continue;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const uint32_t f[4] = {xp[m][0][q][2 * s], xp[m][1][q][2 * s], xp[m][0][q][2 * s + 1], xp[m][1][q][2 * s + 1]};
                    mma16816(sum[m], f, pp[v][2 * s], pp[v][2 * s + 1]);
                }
        }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc(m)[i] += sum[m][i];
}

// The warps' sums, in their order: part[m][j], rows `pitch` apart.
template <int MT, int NT>
__device__ __forceinline__ void add_warps(float (*acc)[NT][4], float *red, float *part, int pitch, int ranks) {
    constexpr int M = 16 * MT, R = 8 * NT;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    __syncthreads();                          // an earlier round's sums have been read
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            float *d = red + (warp * M + 16 * m + g) * (R + 8) + 8 * j + 2 * t;
            *reinterpret_cast<float2 *>(d) = make_float2(acc[m][j][0], acc[m][j][1]);
            *reinterpret_cast<float2 *>(d + 8 * (R + 8)) = make_float2(acc[m][j][2], acc[m][j][3]);
        }
    __syncthreads();
    for (int e = threadIdx.x; e < M * R; e += THREADS) {
        float v[WARPS];
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v[w] = red[(w * M + e / R) * (R + 8) + e % R];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) v[0] += v[w];
        if (e % R < ranks) part[e / R * pitch + e % R] = v[0];
    }
}

// The blocks' parts at p, in their order.
__device__ __forceinline__ float add_blocks(const cg::cluster_group &cluster, float *p, int split) {
    float v[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = split == 1 ? (c == 0 ? *p : 0.0f) : c < split ? *cluster.map_shared_rank(p, c) : 0.0f;
#pragma unroll
    for (int c = 1; c < 8; ++c) v[0] += v[c];
    return v[0];
}

// A launch of clusters of a.split blocks.
cudaError_t launch_clusters(void (*kern)(Args), const Args &a, int64_t tiles, int smem, int most, cudaStream_t s);

// SMALL rows or fewer, one launch.
cudaError_t launch_few(const Args &a, int in_bf16, int p_bf16, cudaStream_t s);

}  // namespace adapters
}  // namespace minw
