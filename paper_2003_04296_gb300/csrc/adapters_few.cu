// adapters_few.cu -- low-rank adapters of a few rows of any users, in one launch.
// Bound by latency: launch, ids, x and down, the sums of a cluster, up, y follow each
// other.  8192 -> 1024 at rank 16, bf16, one row: 5.9 us from the kernel's start to its end
// (ids 0.4, down 1.5, sums 1.2, up and y 2.5), of which 41 ns are its 0.3 MB.
#include "adapters.cuh"

namespace minw {
namespace adapters {

// acc[m][j] += in[rows][k] p1[j][k] over this warp's share of the blocks b0 .. b1 of 32 values: lane t's eight values of a row are
// the operands of two products.  DEPTH blocks are on their way at a time.
template <typename TI, typename TP, bool ODD, int MT, int NT, int DEPTH>
__device__ __forceinline__ void narrow(const Args &a, const int *rows, int count, const TP *p1, int ranks, int b0, int b1,
                                       float (*acc)[NT][4]) {
    constexpr int PI = parts_of<TI>(), PP = parts_of<TP>();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const TI *in = static_cast<const TI *>(a.in);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.0f;
    const TI *row[MT][2];
    bool live[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 16 * m + 8 * i + g;
            live[m][i] = e < count;
            row[m][i] = in + (live[m][i] ? rows[e] : 0) * a.ld_in + 8 * t;
        }
    for (int b = b0 + warp * DEPTH; b < b1; b += WARPS * DEPTH) {
        Eight<TI> x[DEPTH][MT][2];
        Eight<TP> p[DEPTH][NT];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int k = 32 * (b + d), left = b + d < b1 ? a.D - k - 8 * t : 0;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x[d][m][i].template load<ODD>(row[m][i] + k, live[m][i] ? left : 0);
                }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                p[d][j].template load<ODD>(p1 + (int64_t)(8 * j + g) * a.D + k + 8 * t, 8 * j + g < ranks ? left : 0);
            }
        }
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            uint32_t xp[MT][2][PI][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 2; ++i) along(x[d][m][i], xp[m][i]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                uint32_t pp[PP][4];
                along(p[d][j], pp);
                add_products<PI, PP>(xp, pp, [&](int m) { return acc[m][j]; });
            }
        }
    }
}

// Columns 64 b .. + 63 of ME tiles of 16 rows from row m0 of the tile on: h (parts in shared memory, [3][hrows][hpitch]) times the
// user's p2, and the epilogue.  KS steps of 16 of r are loaded at a time.
template <typename TP, bool ODD, int ME, int KS>
__device__ __forceinline__ void widen(const Args &a, const int *rows, int count, int m0, int id, int b, const uint16_t *hs,
                                      int hrows, int hpitch) {
    constexpr int PP = parts_of<TP>();
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    float acc[ME][8][4];
#pragma unroll
    for (int m = 0; m < ME; ++m)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.0f;
    if (id >= 0) {
        const int c = 64 * b + 8 * g, left = a.E - c;
        const TP *p2 = static_cast<const TP *>(a.p2) + (int64_t)id * a.r * a.E + c;
        for (int k0 = 0; k0 < a.rp; k0 += 16 * KS) {
            Eight<TP> p[KS][4];
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = k0 + 16 * s + 2 * t + (i & 1) + 8 * (i >> 1);
                    p[s][i].template load<ODD>(p2 + (int64_t)j * a.E, j < a.r ? left : 0);
                }
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int k = k0 + 16 * s;
                if (k >= a.rp) break;
                uint32_t f[ME][3][4];
#pragma unroll
                for (int m = 0; m < ME; ++m)
#pragma unroll
                    for (int q = 0; q < 3; ++q) {
                        const uint16_t *h = hs + (q * hrows + m0 + 16 * m + g) * hpitch + k + 2 * t;
                        f[m][q][0] = *reinterpret_cast<const uint32_t *>(h);
                        f[m][q][1] = *reinterpret_cast<const uint32_t *>(h + 8 * hpitch);
                        f[m][q][2] = *reinterpret_cast<const uint32_t *>(h + 8);
                        f[m][q][3] = *reinterpret_cast<const uint32_t *>(h + 8 * hpitch + 8);
                    }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint32_t q0[PP], q1[PP];
                    across(p[s][0], p[s][1], i, q0);
                    across(p[s][2], p[s][3], i, q1);
#pragma unroll
                    for (int l = 2; l >= 0; --l)
#pragma unroll
                        for (int q = 0; q <= l; ++q) {
                            const int v = l - q;
                            if (v >= PP) continue;
#pragma unroll
                            for (int m = 0; m < ME; ++m) mma16816(acc[m][i], f[m][q], q0[v], q1[v]);
                        }
                }
            }
        }
    }
    const int c = 64 * b + 16 * t, left = a.E - c;
    if (left > 0) {
#pragma unroll
        for (int m = 0; m < ME; ++m)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int e = m0 + 16 * m + 8 * i + g;
                if (e >= count) continue;
                const int64_t row = rows[e];
                float z[16], f[16];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    z[k] = acc[m][k][2 * i];
                    z[8 + k] = acc[m][k][2 * i + 1];
                }
                if (a.base) {
                    if (a.base_bf16) load16<uint16_t>(a.base, row * a.ld_base + c, left, f);
                    else load16<float>(a.base, row * a.ld_base + c, left, f);
#pragma unroll
                    for (int k = 0; k < 16; ++k) z[k] += f[k];
                }
                if (a.scale || a.shift) {
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (k < left) z[k] = fmaf(z[k], a.scale ? a.scale[c + k] : 1.0f, a.shift ? a.shift[c + k] : 0.0f);
                }
                with_act(a.act, [&](auto act) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) z[k] = act_value<act.value>(z[k]);
                });
                if (a.out_bf16) store16<uint16_t>(a.out, row * a.ld_out + c, left, a.out_vec, z);
                else store16<float>(a.out, row * a.ld_out + c, left, a.out_vec, z);
            }
    }
    __syncwarp();
}

// All of a few rows, one launch: cluster `tile` takes the rows of row `tile`'s user, if it is the first of them, 16 at a time.
template <typename TI, typename TP, int NT, bool ODD>
__global__ void __launch_bounds__(THREADS, 2) few_kernel(const __grid_constant__ Args a) {
    constexpr int R = 8 * NT, BYTES = sizeof(TI) + sizeof(TP), LIMIT = NT == 2 ? 16 / BYTES : NT == 4 ? 8 / BYTES : 1, DEPTH = ODD && LIMIT > 1 ? LIMIT / 2 : LIMIT;
    extern __shared__ __align__(16) uint8_t smem[];
    float *red = reinterpret_cast<float *>(smem);                        // [WARPS][16][R + 8]
    float *part = red + WARPS * 16 * (R + 8);                                  // [SMALL][rp]
    uint16_t *hs = reinterpret_cast<uint16_t *>(part + SMALL * a.rp);    // [3][SMALL][rp + 8]
    __shared__ int all_rows[WARPS][SMALL];                               // each warp finds the rows by itself
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % a.split, tile = blockIdx.x / a.split;
    int *rows = all_rows[warp];
    pdl_wait();
    pdl_trigger();                            // a dependent may rely on what came before this kernel
    const int ids[3] = {a.ids[tile], lane < a.T ? a.ids[lane] : -1, lane + 32 < a.T ? a.ids[lane + 32] : -1};
    const int blocks = (a.D + 31) / 32, b0 = (int)((int64_t)rank * blocks / a.split), b1 = (int)((int64_t)(rank + 1) * blocks / a.split);
    if (b0 + warp * DEPTH + lane < b1 && lane < DEPTH)
        prefetch(static_cast<const TI *>(a.in) + tile * a.ld_in + 32 * (b0 + warp * DEPTH + lane));
    const int mine = user_of(ids[0], a.n), lo = lane < a.T ? user_of(ids[1], a.n) : -1, hi = lane + 32 < a.T ? user_of(ids[2], a.n) : -1;
    const uint32_t ml = __ballot_sync(0xffffffffu, lo == mine), mh = __ballot_sync(0xffffffffu, hi == mine);
    if (tile != (ml ? __ffs(ml) - 1 : 31 + __ffs(mh))) return;           // an earlier row's tile; the whole cluster leaves
    const uint32_t below = (1u << lane) - 1;
    if ((ml >> lane) & 1) rows[__popc(ml & below)] = lane;
    if ((mh >> lane) & 1) rows[__popc(ml) + __popc(mh & below)] = lane + 32;
    __syncwarp();
    const int count = __popc(ml) + __popc(mh), id = mine < a.n ? mine : -1, eblocks = (a.E + 63) / 64;
    // what comes after h, on its way to L2: this warp's columns of p2 and base
    if (id >= 0)
        for (int b = rank * WARPS + warp; b < eblocks; b += a.split * WARPS) {
            constexpr int LINES = 64 * (int)sizeof(TP) / 128, EACH = 128 / (int)sizeof(TP);
            for (int e = lane; e < a.r * LINES; e += 32) {
                const int j = e / LINES, c = 64 * b + e % LINES * EACH;
                if (c < a.E) prefetch(static_cast<const TP *>(a.p2) + ((int64_t)id * a.r + j) * a.E + c);
            }
        }
    if (a.base && 64 * (rank * WARPS + warp) < a.E && lane < count)
        prefetch(static_cast<const uint8_t *>(a.base) + ((int64_t)rows[lane] * a.ld_base + 64 * (rank * WARPS + warp)) * (a.base_bf16 ? 2 : 4));
    cg::cluster_group cluster = cg::this_cluster();
    if (id >= 0) {
        for (int m0 = 0; m0 < count; m0 += 16)
            for (int j0 = 0; j0 < a.r; j0 += R) {
                float acc[1][NT][4];
                narrow<TI, TP, ODD, 1, NT, DEPTH>(a, rows + m0, count - m0, static_cast<const TP *>(a.p1) + ((int64_t)id * a.r + j0) * a.D,
                                             a.r - j0, b0, b1, acc);
                add_warps<1, NT>(acc, red, part + m0 * a.rp + j0, a.rp, a.rp - j0);
            }
        if (a.split > 1) cluster.sync();
        else __syncthreads();
        const float alpha = a.alpha ? a.alpha[id] : 1.0f;
        for (int e = threadIdx.x; e < (count + 15) / 16 * 16 * a.rp; e += THREADS) {
            const float v = add_blocks(cluster, part + e, a.split);
            const int m = e / a.rp, j = e - m * a.rp;
            if (a.h && rank == 0 && m < count && j < a.r) a.h[(int64_t)rows[m] * a.r + j] = v;
            uint32_t s[3];
            split2(__float_as_uint(alpha * v), 0u, s);
#pragma unroll
            for (int q = 0; q < 3; ++q) hs[(q * SMALL + m) * (a.rp + 8) + j] = (uint16_t)s[q];
        }
        __syncwarp();
        if (a.split > 1) cluster_done_reading();
        __syncthreads();
    } else if (rank == 0 && a.h) {
        for (int e = threadIdx.x; e < count * a.r; e += THREADS) a.h[(int64_t)rows[e / a.r] * a.r + e % a.r] = 0.0f;
    }
    constexpr int MOST = (ODD ? 4 : 8) / (int)sizeof(TP), KS = NT / 2 < MOST ? NT / 2 : MOST;
    for (int b = rank * WARPS + warp; b < eblocks; b += a.split * WARPS)
        for (int m0 = 0; m0 < count; m0 += 16) widen<TP, ODD, 1, KS>(a, rows, count, m0, id, b, hs, SMALL, a.rp + 8);
    __syncwarp();
    if (a.split > 1 && id >= 0) cluster_leave();
}

template <typename TI, typename TP, int NT>
static cudaError_t few_of(const Args &a, cudaStream_t s) {
    constexpr int ranks = NT == 8 ? MAX_RANK : 8 * NT;
    auto bytes = [](int rp) { return WARPS * 16 * (8 * NT + 8) * 4 + SMALL * rp * 4 + 3 * SMALL * (rp + 8) * 2; };
    return a.in_vec && a.p1_vec && a.p2_vec ? launch_clusters(few_kernel<TI, TP, NT, false>, a, a.T, bytes(a.rp), bytes(ranks), s)
                                            : launch_clusters(few_kernel<TI, TP, NT, true>, a, a.T, bytes(a.rp), bytes(ranks), s);
}

template <typename TI, typename TP>
static cudaError_t few_types(const Args &a, cudaStream_t s) {
    return a.r <= 16 ? few_of<TI, TP, 2>(a, s) : a.r <= 32 ? few_of<TI, TP, 4>(a, s) : few_of<TI, TP, 8>(a, s);
}

cudaError_t launch_few(const Args &a, int in_bf16, int p_bf16, cudaStream_t s) {
    return in_bf16 ? (p_bf16 ? few_types<uint16_t, uint16_t>(a, s) : few_types<uint16_t, float>(a, s))
                   : (p_bf16 ? few_types<float, uint16_t>(a, s) : few_types<float, float>(a, s));
}

}  // namespace adapters
}  // namespace minw
