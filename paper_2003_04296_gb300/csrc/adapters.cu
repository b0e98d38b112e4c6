// adapters.cu -- low-rank adapters of many requests beside a shared projection:
// row t of user u = ids[t] goes through that user's down [r][K] and up [r][O],
//   h_t = down_u x_t,   y_t = act(scale (base_t + alpha_u up_u^T h_t) + shift)
// and the backward of the term that is added.
//
// Rows of one user share its matrices, so rows are taken in tiles of one user: where a
// tile holds all rows, every tile finds its own (tile t belongs to the first row of its
// user, the others leave) and a cluster takes it: its blocks share the columns of x (K), add
// up their parts of h through each other's shared memory, and share the columns of y (O), one
// launch (adapters_few.cu).  Else a plan sorts the rows by user, and the two products are a launch
// each.  The backward's v_t = alpha_u up_u dy_t, dx_t = down_u^T v_t is the same kernel with the
// matrices exchanged; the matrices' gradients are sums over a user's rows,
//   ddown_u = sum v_t x_t^T,   dup_u = alpha_u sum h_t dy_t^T,   a kernel of their own.
//
// Few operations a value (2 r, r <= 64 as a rule) and short kernels: latency bounds them, and the way of
// instructions that run once.  4096 bf16 rows of 8 users, 4096 -> 4096 at rank 64, 64 us (108 MB: 16 us at the copy rate);
// the backward of 2048 at rank 32, 59.  The products run on mma.sync (bf16; sums over K and over rows in fp32, to nearest, of 32 and 16
// terms each by the tensor cores, which truncate) from registers:
// - along K, the order of the values is free, as long as both operands have the same: a lane
//   takes eight consecutive values of a row for two products of 16;
// - along O (and along K in the gradients), lane g of a group of eight takes eight consecutive columns of
//   rows 2t and 2t + 1 and pairs them up.  Its eight registers are column g of eight products, whose
//   results are 16 consecutive columns a lane.
// fp32 values enter as three bf16 parts (8 + 8 + 8 bits); products of parts below 2^-25 of the
// whole are left out, and where only a bf16 result leaves, those below 2^-16.
#include <math.h>

#include <algorithm>

#include "adapters.cuh"
#include "w4.cuh"

namespace minw {
namespace adapters {

// ---------------------------------------------------------------------------
// The plan
// ---------------------------------------------------------------------------

constexpr int PLAN_THREADS = 1024, PLAN_WARPS = 32;
constexpr int COUNTS = PLAN_WARPS + 1;       // of a user; odd, so that a warp's users lie in different banks

// A warp counts a run of rows, then places them; between the two, the counts [user][warp] become places.  One block:
// 4096 rows are 4 rounds of a warp.
__global__ void __launch_bounds__(PLAN_THREADS) plan_kernel(const int *__restrict__ ids, int T, int n, int most, Plan p,
                                                            int in_shared) {
    pdl_trigger();
    pdl_wait();
    extern __shared__ int counts_smem[];
    int *counts = in_shared ? counts_smem : p.counts;
    __shared__ int warp_rows[PLAN_WARPS], warp_tiles[PLAN_WARPS], base_rows, base_tiles;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int seg = ((T + PLAN_WARPS - 1) / PLAN_WARPS + 31) / 32 * 32;
    const int t0 = min(T, warp * seg), t1 = min(T, t0 + seg);
    for (int k = threadIdx.x; k < (n + 1) * COUNTS; k += PLAN_THREADS) counts[k] = 0;
    if (threadIdx.x == 0) base_rows = base_tiles = 0;
    __syncthreads();
    for (int t = t0 + lane; t - lane < t1; t += 32) {
        const int u = t < t1 ? user_of(ids[t], n) : -1;
        const uint32_t m = __match_any_sync(0xffffffffu, u);
        if (u >= 0 && lane == __ffs(m) - 1) counts[u * COUNTS + warp] += __popc(m);
        __syncwarp();
    }
    __syncthreads();
    for (int u0 = 0; u0 <= n; u0 += PLAN_THREADS) {
        const int u = u0 + threadIdx.x;
        int rows = 0;
        if (u <= n)
            for (int w = 0; w < PLAN_WARPS; ++w) {
                const int c = counts[u * COUNTS + w];
                counts[u * COUNTS + w] = rows;
                rows += c;
            }
        const int tiles = (rows + most - 1) / most;
        int ir = rows, it = tiles;                             // inclusive sums over the block
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int a = __shfl_up_sync(0xffffffffu, ir, d), b = __shfl_up_sync(0xffffffffu, it, d);
            if (lane >= d) { ir += a; it += b; }
        }
        if (lane == 31) { warp_rows[warp] = ir; warp_tiles[warp] = it; }
        __syncthreads();
        int start = base_rows + ir - rows, tile = base_tiles + it - tiles;
        for (int w = 0; w < warp; ++w) { start += warp_rows[w]; tile += warp_tiles[w]; }
        if (u <= n) {
            p.first[u] = start;
            for (int w = 0; w < PLAN_WARPS; ++w) counts[u * COUNTS + w] += start;
            for (int k = 0; k < tiles; ++k)
                p.tiles[tile + k] = Tile{u < n ? u : -1, start + k * most, min(most, rows - k * most), 0};
        }
        __syncthreads();
        if (threadIdx.x == PLAN_THREADS - 1) { base_rows = start + rows; base_tiles = tile + tiles; }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        p.first[n + 1] = T;
        *p.tiles_n = base_tiles;
    }
    for (int t = t0 + lane; t - lane < t1; t += 32) {
        const int u = t < t1 ? user_of(ids[t], n) : -1;
        const uint32_t m = __match_any_sync(0xffffffffu, u);
        int at = 0;
        if (u >= 0) at = counts[u * COUNTS + warp] + __popc(m & ((1u << lane) - 1));
        __syncwarp();
        if (u >= 0) {
            p.order[at] = t;
            if (lane == __ffs(m) - 1) counts[u * COUNTS + warp] += __popc(m);
        }
        __syncwarp();
    }
}

// ---------------------------------------------------------------------------
// Through an adapter
// ---------------------------------------------------------------------------

// `bytes` (16) to shared memory, asynchronously, the first `n` of them from src and zeros behind.
__device__ __forceinline__ void copy_fill(uint32_t dst, const void *src, int n) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}

// A warp's eights on their way through shared memory: 16 bytes a lane (fp32: twice).  ODD: rows lie off 16-byte boundaries.  Then
// the aligned sixteens are copied that hold values of the row, and a lane's eight is shifted out of its own and the first
// of the lane `next` behind; the last of these copies one more, to the end.
template <typename V, bool ODD>
struct Way {
    static constexpr int C = (int)sizeof(V) / 2, BYTES = C * 512 + (ODD ? 128 : 0);

    // p: the lane's eight, left: values of the row from there on (few or none: zeros).  spare: the last lane's place at the end, else -1.
    static __device__ __forceinline__ void fetch(uint32_t item, const V *p, int left, const void *safe, int spare) {
        const int lane = threadIdx.x & 31;
        if constexpr (!ODD) {
            constexpr int N = 8 / C;                                     // values in 16 bytes
#pragma unroll
            for (int h = 0; h < C; ++h) {
                const int n = min(max(left - h * N, 0), N);
                copy_fill(item + lane * 16 + 512 * h, n > 0 ? p + h * N : safe, n * (int)sizeof(V));
            }
        } else {
            const int64_t at = (int64_t)reinterpret_cast<uintptr_t>(p), first = at & ~(int64_t)15, end = at + (int64_t)left * (int)sizeof(V);
            safe = reinterpret_cast<const void *>(reinterpret_cast<uintptr_t>(safe) & ~(uintptr_t)15);      // a copy of no bytes has to be aligned, too
#pragma unroll
            for (int h = 0; h < C; ++h)
                copy_fill(item + lane * 16 + 512 * h, first + 16 * h < end ? reinterpret_cast<const void *>(first + 16 * h) : safe,
                          first + 16 * h < end ? 16 : 0);
            if (spare >= 0)
                copy_fill(item + C * 512 + spare * 16, first + 16 * C < end ? reinterpret_cast<const void *>(first + 16 * C) : safe,
                          first + 16 * C < end ? 16 : 0);
        }
    }
    // off: the row's distance from a 16-byte boundary
    static __device__ __forceinline__ void read(uint32_t item, Eight<V> &e, int left, int off, int next, int spare) {
        const int lane = threadIdx.x & 31;
        uint32_t u[4 * C + 4];
#pragma unroll
        for (int h = 0; h < C + (ODD ? 1 : 0); ++h) {
            const uint32_t at = h < C ? item + lane * 16 + 512 * h : spare >= 0 ? item + C * 512 + spare * 16 : item + (lane + next) * 16;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(u[4 * h]), "=r"(u[4 * h + 1]), "=r"(u[4 * h + 2]), "=r"(u[4 * h + 3])
                         : "r"(at)
                         : "memory");
        }
        if constexpr (ODD) shifted<4 * C>(u, off);
#pragma unroll
        for (int k = 0; k < 4 * C; ++k) e.w[k] = u[k];
        if constexpr (ODD) e.cut(left);
    }
};

// 8 rows of 64 columns, 16 a lane (row lane / 4, columns 16 (lane % 4) on), to rows anywhere: through shared memory, laid out as
// the row lies to 16-byte boundaries, and from there by sixteens (a value at a time from here: 32 sectors an instruction).
// row: this lane's row at the first of the columns, null for none.  n: columns of the row.
template <typename V>
__device__ __forceinline__ void put8(V *stage, const float *v, V *row, int n) {
    constexpr int PITCH = 72, E = 16 / (int)sizeof(V), CHUNKS = PITCH / E;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int off = (int)(reinterpret_cast<uintptr_t>(row) & 15) / (int)sizeof(V);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        Vec<V, 1> w;
        w.set(v + k);
        w.store(stage + g * PITCH + off + 16 * t + k);
    }
    __syncwarp();
#pragma unroll 1
    for (int e0 = 0; e0 < 8 * CHUNKS; e0 += 32) {
        const int e = e0 + lane, r = min(e / CHUNKS, 7), c = (e - r * CHUNKS) * E;
        V *to = reinterpret_cast<V *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), 4 * r));
        const int o = (int)(reinterpret_cast<uintptr_t>(to) & 15) / (int)sizeof(V), first = max(c, o), last = min(c + E, o + n);
        if (e >= 8 * CHUNKS || !to || first >= last) continue;
        const V *from = stage + r * PITCH;
        if (last - first == E) *reinterpret_cast<uint4 *>(to - o + c) = *reinterpret_cast<const uint4 *>(from + c);
        else
            for (int k = first; k < last; ++k) to[k - o] = from[k];
    }
    __syncwarp();
}
constexpr int STAGE_BYTES = 8 * 72 * 4;

__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint32_t shared_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Where value j (of 16) of a row of h lies in its parts: the four that lane t of a product takes, 2t, 2t + 1, 2t + 8, 2t + 9,
// side by side.
__device__ __forceinline__ int place(int j) { return ((j & 7) >> 1) * 4 + (j >> 3) * 2 + (j & 1); }
__device__ __forceinline__ int value_at(int p) { return 2 * (p >> 2) + (p & 1) + 8 * ((p >> 1) & 1); }

// What the kernels below have on its way: a warp copies units of what it will work on next into a ring of its own in shared
// memory, and a lane reads back what it has copied itself, without a barrier.  (The same loads into registers, two
// blocks of 8 warps an SM: 35 and 67 us for the two halves of 4096 rows, 4096 -> 4096 at rank 64.)

template <typename TI, typename TP, int MT, int NT, bool ODD>
struct NarrowRing {
    static constexpr int UNIT = MT * 2 * Way<TI, ODD>::BYTES + NT * Way<TP, ODD>::BYTES;           // 32 values along D
    static constexpr int DEPTH = 220 * 1024 / (WARPS * UNIT) < 4 ? 220 * 1024 / (WARPS * UNIT) : 4;
    static constexpr int BYTES = WARPS * DEPTH * UNIT;
    static_assert(DEPTH >= 2 && BYTES >= 16 * MT * (WARPS * (8 * NT + 8) + 8 * NT) * 4, "the sums lie where the ring was");
};

// The plan's tiles, first half: h, and alpha h in parts for the second half and the gradients.
template <typename TI, typename TP, int MT, int NT, bool ODD>
__global__ void __launch_bounds__(THREADS, 1) narrow_kernel(const __grid_constant__ Args a) {
    constexpr int M = 16 * MT, R = 8 * NT, PI = parts_of<TI>(), PP = parts_of<TP>();
    using Ring = NarrowRing<TI, TP, MT, NT, ODD>;
    using In = Way<TI, ODD>;
    using Pool = Way<TP, ODD>;
    extern __shared__ __align__(16) uint8_t smem[];
    float *red = reinterpret_cast<float *>(smem);                        // [WARPS][M][R + 8], when the ring is done with
    float *part = red + WARPS * M * (R + 8);                             // [M][R]
    __shared__ int rows[M];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rank = blockIdx.x % a.split, tile = blockIdx.x / a.split;
    const uint32_t ring = shared_at(smem) + warp * Ring::DEPTH * Ring::UNIT;
    const int spare = t == 3 ? g : -1;
    pdl_wait();
    pdl_trigger();
    const int tiles = *a.plan.tiles_n;
    const Tile x = a.plan.tiles[tile];                                   // there is room for as many as blocks
    if (tile >= tiles) return;
    if (threadIdx.x < x.count) rows[threadIdx.x] = a.plan.order[x.start + threadIdx.x];
    __syncthreads();
    if (x.id < 0) {
        if (rank == 0 && a.h)
            for (int e = threadIdx.x; e < x.count * a.r; e += THREADS) a.h[(int64_t)rows[e / a.r] * a.r + e % a.r] = 0.0f;
        return;
    }
    cg::cluster_group cluster = cg::this_cluster();
    const float alpha = a.alpha ? a.alpha[x.id] : 1.0f;
    const int blocks = (a.D + 31) / 32, b0 = (int)((int64_t)rank * blocks / a.split), b1 = (int)((int64_t)(rank + 1) * blocks / a.split);
    const TI *row[MT][2];
    bool live[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 16 * m + 8 * i + g;
            live[m][i] = e < x.count;
            row[m][i] = static_cast<const TI *>(a.in) + (live[m][i] ? rows[e] : rows[0]) * a.ld_in + 8 * t;
        }
    for (int j0 = 0; j0 < a.r; j0 += R) {
        const TP *p1 = static_cast<const TP *>(a.p1) + ((int64_t)x.id * a.r + j0) * a.D + 8 * t;
        int next = b0 + warp, put = 0, get = 0;
        auto fetch = [&]() {
            if (next < b1) {
                const uint32_t d = ring + put * Ring::UNIT;
                const int k = 32 * next, left = a.D - k - 8 * t;
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        In::fetch(d + (2 * m + i) * In::BYTES, row[m][i] + k, live[m][i] ? left : -8, a.in, spare);
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    Pool::fetch(d + 2 * MT * In::BYTES + j * Pool::BYTES, p1 + (int64_t)(8 * j + g) * a.D + k,
                                j0 + 8 * j + g < a.r ? left : -8, a.p1, spare);
            }
            commit();
            next += WARPS;
            if (++put == Ring::DEPTH) put = 0;
        };
#pragma unroll
        for (int d = 0; d < Ring::DEPTH - 1; ++d) fetch();
        float acc[MT][NT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.0f;
        for (int b = b0 + warp; b < b1; b += WARPS) {
            arrived<Ring::DEPTH - 2>();
            if (ODD) __syncwarp();                                       // the neighbours' too; and they have read the slot that comes next
            fetch();
            const uint32_t d = ring + get * Ring::UNIT;
            if (++get == Ring::DEPTH) get = 0;
            const int left = a.D - 32 * b - 8 * t;
            uint32_t xp[MT][2][PI][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    Eight<TI> e;
                    In::read(d + (2 * m + i) * In::BYTES, e, left, (int)(reinterpret_cast<uintptr_t>(row[m][i]) & 15), 1, spare);
                    along(e, xp[m][i]);
                }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                Eight<TP> e;
                uint32_t pp[PP][4];
                Pool::read(d + 2 * MT * In::BYTES + j * Pool::BYTES, e, left,
                           (int)(reinterpret_cast<uintptr_t>(p1 + (int64_t)(8 * j + g) * a.D) & 15), 1, spare);
                along(e, pp);
                add_products<PI, PP>(xp, pp, [&](int m) { return acc[m][j]; });
            }
        }
        arrived<0>();
        add_warps<MT, NT>(acc, red, part, R, R);
        if (a.split > 1) cluster.sync();
        else __syncthreads();
        // a block finishes its share of the rows
        const int each = (M + a.split - 1) / a.split, e1 = min(x.count, (rank + 1) * each) * R;
        for (int e = rank * each * R + threadIdx.x; e < e1; e += THREADS) {
            const int m = e / R, j = j0 + e % R;
            if (j >= a.rp) continue;
            const float v = add_blocks(cluster, part + e, a.split);
            const int64_t at = (int64_t)(x.start + m) * a.rp + j / 16 * 16 + place(j & 15);
            uint32_t s[3];
            split2(__float_as_uint(alpha * v), 0u, s);
#pragma unroll
            for (int q = 0; q < 3; ++q) a.hp[(int64_t)q * a.T * a.rp + at] = (uint16_t)s[q];
            if (a.h && j < a.r) a.h[(int64_t)rows[m] * a.r + j] = v;
            if (a.hh) {
                split2(__float_as_uint(j < a.r ? alpha * a.h_in[(int64_t)rows[m] * a.r + j] : 0.0f), 0u, s);
#pragma unroll
                for (int q = 0; q < 3; ++q) a.hh[(int64_t)q * a.T * a.rp + at] = (uint16_t)s[q];
            }
        }
        // before the next round's ring lies where the parts are
        if (j0 + R < a.r) {
            if (a.split > 1) cluster.sync();
            else __syncthreads();
        }
    }
    if (a.split > 1) {
        __syncwarp();
        cluster_done_reading();
        cluster_leave();
    }
}

// A lane's four rows of 16 columns, c the first: base added, for whole blocks on 16-byte boundaries.
template <typename V>
__device__ __forceinline__ void add16(const Args &a, const int (*rows)[2], int c, float (*acc)[8][4]) {
    Vec<V, 8> w[2][2][2];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const V *p = static_cast<const V *>(a.base) + (int64_t)max(rows[m][i], 0) * a.ld_base + c;
            w[m][i][0].load(p);
            w[m][i][1].load(p + 8);
        }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[m][k & 7][2 * i + (k >> 3)] += w[m][i][k >> 3].get(k & 7);
}

// ... and the result, n columns of a block of 64.
template <typename V>
__device__ __forceinline__ void put16(const Args &a, const int (*rows)[2], int c, int n, const float (*acc)[8][4], uint8_t *stage) {
    const bool whole = a.out_vec && n == 64;
    if (whole) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float v[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = acc[m][k & 7][2 * i + (k >> 3)];
                V *row = static_cast<V *>(a.out) + (int64_t)max(rows[m][i], 0) * a.ld_out + c;
                if (rows[m][i] >= 0) {
                    Vec<V, 8> w;
                    w.set(v);
                    w.store(row);
                    w.set(v + 8);
                    w.store(row + 8);
                }
            }
    } else {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float v[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = acc[m][k & 7][2 * i + (k >> 3)];
                put8(reinterpret_cast<V *>(stage), v,
                     rows[m][i] >= 0 ? static_cast<V *>(a.out) + (int64_t)rows[m][i] * a.ld_out + c - 16 * (threadIdx.x & 3) : nullptr, n);
            }
    }
}

template <typename TP, bool ODD>
struct WidenRing {
    static constexpr int UNIT = 4 * Way<TP, ODD>::BYTES, DEPTH = sizeof(TP) == 2 ? 4 : 2;      // 16 of r x 64 columns
};

// ... second half: a block takes `per` blocks of 64 columns of a tile, a warp at a time one of them for 32 rows.  h lies in shared
// memory for all warps, p2 comes by a warp's ring.
template <typename TP, bool FINE, bool ODD>
__global__ void __launch_bounds__(THREADS, 2) widen_kernel(const __grid_constant__ Args a, int groups, int per) {
    constexpr int PP = parts_of<TP>(), PARTS = FINE ? 3 : 2;
    using Ring = WidenRing<TP, ODD>;
    using Pool = Way<TP, ODD>;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int rows[64];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int steps = a.rp / 16, hpitch = a.rp + 8;
    const uint32_t ring = shared_at(smem) + warp * (Ring::DEPTH * Ring::UNIT);
    const int spare = g == 7 ? t : -1;
    uint8_t *stage = smem + WARPS * Ring::DEPTH * Ring::UNIT + warp * STAGE_BYTES;
    const uint16_t *hs = reinterpret_cast<uint16_t *>(smem + WARPS * (Ring::DEPTH * Ring::UNIT + STAGE_BYTES));      // [PARTS][most][hpitch]
    const int tile = blockIdx.x / groups, first = (blockIdx.x - tile * groups) * per, last = min((a.E + 63) / 64, first + per);
    pdl_wait();
    pdl_trigger();                            // the gradients rely on what came before this kernel
    const int tiles = *a.plan.tiles_n;
    const Tile x = a.plan.tiles[tile];
    if (tile >= tiles) return;
    const int halves = x.count > 32 ? 2 : 1, blocks = max(0, (last - first - warp + WARPS - 1) / WARPS);
    // this warp's units: blocks first + warp, first + warp + WARPS, ..., their halves, steps along r
    const int units = x.id >= 0 ? blocks * halves * steps : 0;
    const TP *p2 = static_cast<const TP *>(a.p2) + (int64_t)max(x.id, 0) * a.r * a.E;
    int put = 0, next = 0, next_b = first + warp, next_h = 0, next_s = 0;
    auto fetch = [&]() {
        if (next < units) {
            const int c = 64 * next_b + 8 * g, left = a.E - c;
            const uint32_t d = ring + put * Ring::UNIT;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = 16 * next_s + 2 * t + (e & 1) + 8 * (e >> 1);
                Pool::fetch(d + e * Pool::BYTES, p2 + (int64_t)min(j, a.r - 1) * a.E + c, j < a.r ? left : -1000, a.p2, spare);
            }
            ++next;
            if (++next_s == steps) {
                next_s = 0;
                if (++next_h == halves) {
                    next_h = 0;
                    next_b += WARPS;
                }
            }
        }
        commit();
        put = (put + 1) % Ring::DEPTH;
    };
    if (threadIdx.x < x.count) rows[threadIdx.x] = a.plan.order[x.start + threadIdx.x];
    if (x.id >= 0) {
        const int eights = a.rp / 8;
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
            for (int e = threadIdx.x; e < a.most * eights; e += THREADS) {
                const int m = e / eights, j = 8 * (e - m * eights);
                copy_fill(shared_at(hs + (q * a.most + m) * hpitch + j),
                              a.hp + ((int64_t)q * a.T + x.start + min(m, x.count - 1)) * a.rp + j, m < x.count ? 16 : 0);
            }
        commit();
#pragma unroll
        for (int d = 0; d < Ring::DEPTH - 1; ++d) fetch();
        arrived<Ring::DEPTH - 1>();
    }
    __syncthreads();
    int get = 0;
    for (int u = 0; u < blocks * halves; ++u) {
        const int h = halves == 2 ? u & 1 : 0, b = first + warp + (u / halves) * WARPS;
        const int c = 64 * b + 16 * t, left = a.E - c;
        int row[2][2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int e = 32 * h + 16 * m + 8 * i + g;
                row[m][i] = e < x.count ? rows[e] : -1;
                if (a.base && left > 0 && row[m][i] >= 0)                // on its way to L2 during the products
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint8_t *>(a.base) +
                                                                   ((int64_t)row[m][i] * a.ld_base + c) * (a.base_bf16 ? 2 : 4)));
            }
        float acc[2][8][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.0f;
        if (x.id >= 0)
#pragma unroll 1
            for (int step = 0; step < steps; ++step) {
                if (ODD) __syncwarp();
                fetch();                                                 // where the last one read was
                arrived<Ring::DEPTH - 1>();
                if (ODD) __syncwarp();
                const uint32_t d = ring + get * Ring::UNIT;
                get = (get + 1) % Ring::DEPTH;
                Eight<TP> p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = 16 * step + 2 * t + (i & 1) + 8 * (i >> 1);
                    Pool::read(d + i * Pool::BYTES, p[i], a.E - 64 * b - 8 * g,
                               (int)(reinterpret_cast<uintptr_t>(p2 + (int64_t)min(j, a.r - 1) * a.E) & 15), 4, spare);
                }
                uint32_t f[2][3][4];
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int q = 0; q < PARTS; ++q)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint2 w = *reinterpret_cast<const uint2 *>(
                                hs + (q * a.most + 32 * h + 16 * m + 8 * i + g) * hpitch + 16 * step + 4 * t);
                            f[m][q][i] = w.x;
                            f[m][q][2 + i] = w.y;
                        }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint32_t q0[PP], q1[PP];
                    across(p[0], p[1], i, q0);
                    across(p[2], p[3], i, q1);
#pragma unroll
                    for (int l = 2; l >= 0; --l)
#pragma unroll
                        for (int q = 0; q <= l; ++q) {
                            const int v = l - q;
                            if (v >= PP || (l == 2 && !FINE)) continue;
#pragma unroll
                            for (int m = 0; m < 2; ++m) mma16816(acc[m][i], f[m][q], q0[v], q1[v]);
                        }
                }
            }
        // value k of the lane's 16 of row (m, i)
        auto z = [&](int m, int i, int k) -> float & { return acc[m][k & 7][2 * i + (k >> 3)]; };
        // Whole blocks on 16-byte boundaries by themselves: with the other way inlined beside each load, the instructions come late.
        const bool whole = 64 * b + 64 <= a.E;
        if (a.base && a.base_vec && whole) {
            if (a.base_bf16) add16<uint16_t>(a, row, c, acc);
            else add16<float>(a, row, c, acc);
        } else if (a.base) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float f[16];
                    const int64_t at = (int64_t)max(row[m][i], 0) * a.ld_base + c;
                    const int n = row[m][i] >= 0 ? left : 0;
                    if (a.base_bf16) load16<uint16_t>(a.base, at, n, f);
                    else load16<float>(a.base, at, n, f);
#pragma unroll
                    for (int k = 0; k < 16; ++k) z(m, i, k) += f[k];
                }
        }
        if (a.scale || a.shift) {
#pragma unroll
            for (int k0 = 0; k0 < 16; k0 += 4) {
                float sc[4] = {1.0f, 1.0f, 1.0f, 1.0f}, sh[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (a.scale_vec && whole) {
                    if (a.scale) *reinterpret_cast<float4 *>(sc) = *reinterpret_cast<const float4 *>(a.scale + c + k0);
                    if (a.shift) *reinterpret_cast<float4 *>(sh) = *reinterpret_cast<const float4 *>(a.shift + c + k0);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k0 + k < left) {
                            if (a.scale) sc[k] = a.scale[c + k0 + k];
                            if (a.shift) sh[k] = a.shift[c + k0 + k];
                        }
                }
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int k = 0; k < 4; ++k) z(m, i, k0 + k) = fmaf(z(m, i, k0 + k), sc[k], sh[k]);
            }
        }
        if (a.act != MINW_ACT_NONE)
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k) z(m, i, k) = act_value<act.value>(z(m, i, k));
            });
        if (a.out_bf16) put16<uint16_t>(a, row, c, min(64, a.E - 64 * b), acc, stage);
        else put16<float>(a, row, c, min(64, a.E - 64 * b), acc, stage);
        __syncwarp();
    }
}

// ---------------------------------------------------------------------------
// Gradients of the matrices: out_u [r][C] = sum over rows of u of a[j][place] z[row][c]
// ---------------------------------------------------------------------------

struct Job {
    const uint16_t *a;                       // [3][T][rp] by sorted row, in parts
    const void *z;                           // [T][C], rows ld apart
    float *out;                              // [n][r][C]
    int64_t ld;
    int C, blocks;                           // blocks: of this job for a user
    int odd, out_vec;                        // z, out: rows off 16-byte boundaries, on them
};

struct GradArgs {
    Job job[2];
    int jobs, T, n, r, rp, along;            // along: warps that share a user's rows (the others: columns)
    int beside;                              // the kernel before this one makes dx
    Plan plan;
};

constexpr int CHUNK = 64;                    // rows whose parts are in shared memory at a time
constexpr int ORDER = 1024;                  // rows whose places are

template <typename TZ, int RT, bool ODD>
struct GradRing {
    static constexpr int UNIT = 4 * Way<TZ, ODD>::BYTES, DEPTH = sizeof(TZ) == 2 ? 4 : 2, BYTES = WARPS * DEPTH * UNIT;
    static constexpr int PITCH = 16 * RT + 8, PARTS = 3 * CHUNK * PITCH * 2;       // bytes of a chunk's parts, twice
    static constexpr int ALL = BYTES + (2 * PARTS > WARPS * STAGE_BYTES ? 2 * PARTS : WARPS * STAGE_BYTES);
};

// RT: tiles of 16 of r in one go.  A warp takes 64 columns: its rows' values come by a ring of its own (as above), the parts of the
// rows, which all warps need, by chunks for the block.
template <typename TZ, int RT, bool ODD>
__global__ void __launch_bounds__(THREADS, RT < 4 ? 2 : 1) grads_kernel(const __grid_constant__ GradArgs a) {
    constexpr int PZ = parts_of<TZ>();
    using Ring = GradRing<TZ, RT, ODD>;
    using Row = Way<TZ, ODD>;
    extern __shared__ __align__(16) uint8_t smem[];
    float *red = reinterpret_cast<float *>(smem);                        // [WARPS][16][64] where warps share rows
    uint8_t *parts = smem + Ring::BYTES;                                 // [2][3][CHUNK][PITCH]
    __shared__ int order[ORDER];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int all = a.job[0].blocks + (a.jobs > 1 ? a.job[1].blocks : 0);
    const int u = blockIdx.x / all;
    int b = blockIdx.x - u * all;
    const Job &job = a.job[b >= a.job[0].blocks ? 1 : 0];
    if (b >= a.job[0].blocks) b -= a.job[0].blocks;
    const int wa = warp % a.along, wc = warp / a.along;
    const int c0 = 64 * (b * (WARPS / a.along) + wc), c = c0 + 8 * g, left = job.C - c;
    const uint32_t ring = shared_at(smem) + warp * Ring::DEPTH * Ring::UNIT;
    const int spare = g == 7 ? t : -1;
    const TZ *z = static_cast<const TZ *>(job.z);
    pdl_trigger();
    // Beside the kernel that makes dx, whose results are not needed here: it lets this one start once the parts are there, and is
    // waited for at the end, for those who wait for this one.  Until then all that earlier kernels wrote is read through L2, where it
    // lay before that one let this one start: what an SM's own cache holds is certain to be new only after a wait.
    if (!a.beside) pdl_wait();
    const int first = __ldcg(a.plan.first + u), count = __ldcg(a.plan.first + u + 1) - first;
    for (int j0 = 0; j0 < a.r; j0 += 16 * RT) {
        float acc[RT][8][4];
#pragma unroll
        for (int m = 0; m < RT; ++m)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[m][i][k] = 0.0f;
        const int ranks = min(16 * RT, a.rp - j0);
        for (int s0 = 0; s0 < count; s0 += ORDER) {
            const int seg = min(ORDER, count - s0);
            __syncthreads();
            for (int e = threadIdx.x; e < seg; e += THREADS) order[e] = __ldcg(a.plan.order + first + s0 + e);
            __syncthreads();
            // the warp's steps of 16 rows: wa, wa + along, ...
            int next = wa, put = 0, get = 0;
            auto fetch = [&]() {
                if (16 * next < seg) {
                    const uint32_t d = ring + put * Ring::UNIT;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int e = 16 * next + 2 * t + (i & 1) + 8 * (i >> 1);
                        Row::fetch(d + i * Row::BYTES, z + order[min(e, seg - 1)] * job.ld + c, e < seg ? left : -1000, z, spare);
                    }
                }
                next += a.along;
                if (++put == Ring::DEPTH) put = 0;
            };
            auto fetch_parts = [&](int chunk) {                          // rows past the last: zeros
                constexpr int EIGHTS = 2 * RT;
                const int rows0 = chunk * CHUNK;
                if (rows0 < seg)
                    for (int e = threadIdx.x; e < 3 * CHUNK * EIGHTS; e += THREADS) {
                        const int q = e / (CHUNK * EIGHTS), m = e / EIGHTS % CHUNK, j = 8 * (e % EIGHTS);
                        if (j >= ranks) continue;
                        const bool some = rows0 + m < seg;
                        copy_fill(shared_at(parts + (chunk & 1) * Ring::PARTS + ((q * CHUNK + m) * Ring::PITCH + j) * 2),
                                      job.a + ((int64_t)q * a.T + first + s0 + (some ? rows0 + m : 0)) * a.rp + j0 + j, some ? 16 : 0);
                    }
            };
            fetch_parts(0);
            commit();
#pragma unroll
            for (int d = 0; d < Ring::DEPTH - 1; ++d) {
                fetch();
                commit();
            }
            for (int chunk = 0; chunk * CHUNK < seg; ++chunk) {
                // the chunk's parts went out before the units of the chunk before (the first one's: of the whole ring)
                if (a.along == 1) arrived<Ring::DEPTH - 1>();            // (at most four)
                else if (a.along == 2) arrived<(Ring::DEPTH > 2 ? 2 : 1)>();
                else arrived<1>();
                __syncthreads();
                fetch_parts(chunk + 1);
                commit();
#pragma unroll 1
                for (int s = wa; s < CHUNK / 16; s += a.along) {         // (along divides a chunk's steps)
                    const int step = chunk * (CHUNK / 16) + s;
                    if (16 * step >= seg) break;
                    if (ODD) __syncwarp();
                    fetch();
                    commit();
                    arrived<Ring::DEPTH - 1>();
                    if (ODD) __syncwarp();
                    const uint32_t d = ring + get * Ring::UNIT;
                    if (++get == Ring::DEPTH) get = 0;
                    Eight<TZ> v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int e = 16 * step + 2 * t + (i & 1) + 8 * (i >> 1);
                        const int off = ODD ? (int)(reinterpret_cast<uintptr_t>(z + order[min(e, seg - 1)] * job.ld) & 15) : 0;
                        Row::read(d + i * Row::BYTES, v[i], left, off, 4, spare);
                    }
                    uint32_t f[RT][3][4];
#pragma unroll
                    for (int m = 0; m < RT; ++m)
#pragma unroll
                        for (int q = 0; q < 3; ++q) {
                            // four transposed 8 x 8 pieces: rows 0-7 and 8-15 of both halves of j
                            const uint32_t at = shared_at(parts + (chunk & 1) * Ring::PARTS) +
                                                ((q * CHUNK + 16 * s + (lane & 7) + 8 * (lane >> 4)) * Ring::PITCH + 16 * m + 8 * ((lane >> 3) & 1)) * 2;
                            asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(f[m][q][0]), "=r"(f[m][q][1]), "=r"(f[m][q][2]), "=r"(f[m][q][3])
                                         : "r"(at)
                                         : "memory");
                        }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint32_t q0[PZ], q1[PZ];
                        across(v[0], v[1], i, q0);
                        across(v[2], v[3], i, q1);
                        float sum[RT][4];                                // 16 rows, then to nearest into all rows' sums
#pragma unroll
                        for (int m = 0; m < RT; ++m)
#pragma unroll
                            for (int k = 0; k < 4; ++k) sum[m][k] = 0.0f;
#pragma unroll
                        for (int l = 2; l >= 0; --l)
#pragma unroll
                            for (int q = 0; q <= l; ++q) {
                                const int k = l - q;
                                if (k >= PZ) continue;
#pragma unroll
                                for (int m = 0; m < RT; ++m) mma16816(sum[m], f[m][q], q0[k], q1[k]);
                            }
#pragma unroll
                        for (int m = 0; m < RT; ++m)
#pragma unroll
                            for (int k = 0; k < 4; ++k) acc[m][i][k] += sum[m][k];
                    }
                }
                __syncthreads();                                         // the parts have been read
            }
            arrived<0>();
        }
        __syncthreads();                      // results are staged where the parts were
#pragma unroll
        for (int m = 0; m < RT; ++m) {
            if (a.along > 1) {                // the warps of a column block in their order, into the first
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) red[(warp * 32 + 4 * i + k) * 32 + lane] = acc[m][i][k];
                __syncthreads();
                if (wa == 0)
                    for (int w = 1; w < a.along; ++w)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
#pragma unroll
                            for (int k = 0; k < 4; ++k) acc[m][i][k] += red[((warp + w) * 32 + 4 * i + k) * 32 + lane];
            }
            if (wa != 0) continue;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int j = j0 + 16 * m + value_at(8 * i + g);
                float y[16];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    y[k] = acc[m][k][2 * i];
                    y[8 + k] = acc[m][k][2 * i + 1];
                }
                float *row = j < a.r ? job.out + ((int64_t)u * a.r + j) * job.C + c0 : nullptr;
                if (c0 >= job.C) continue;
                if (!job.out_vec || job.C - c0 < 64) put8(reinterpret_cast<float *>(parts + warp * STAGE_BYTES), y, row, min(64, job.C - c0));
                else if (row) store16<float>(row, 16 * t, 16, true, y);
            }
        }
        __syncthreads();
    }
    if (a.beside) pdl_wait();
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

using namespace minw_host;

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Rows of a tile: 64, where h in registers (and a ring in shared memory) leaves room for them, else 32.
static int rows_of(int r, bool bf16) { return r <= 32 || (r <= 64 && bf16) ? 64 : 32; }
static int rank_pitch(int r) { return (r + 15) / 16 * 16; }

constexpr int W4_ROWS = 32;                  // rows of w4 products at a time
static int64_t w4_bytes(int64_t T, int O) { return std::min<int64_t>(T, W4_ROWS) * O * 4; }       // their adapters' terms

static int64_t tiles_of(int64_t T, int n, int most) { return std::min<int64_t>(T, T / most + std::min<int64_t>(T, (int64_t)n + 1)); }

static bool counts_in_shared(int n) { return (int64_t)(n + 1) * COUNTS * 4 <= 128 * 1024; }

static Plan plan_at(uint8_t *base, int64_t T, int n, int r, int64_t *used) {
    Plan p;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        uint8_t *q = base + at;
        at += up(bytes, 16);
        return q;
    };
    p.tiles = reinterpret_cast<Tile *>(take(tiles_of(T, n, rows_of(r, false)) * sizeof(Tile)));
    p.order = reinterpret_cast<int *>(take(T * 4));
    p.first = reinterpret_cast<int *>(take(((int64_t)n + 2) * 4));
    p.tiles_n = reinterpret_cast<int *>(take(4));
    p.counts = reinterpret_cast<int *>(take(counts_in_shared(n) ? 0 : ((int64_t)n + 1) * COUNTS * 4));
    *used = at;
    return p;
}

static minw_status make_plan(const Plan &p, const int *ids, int T, int n, int most, cudaStream_t s) {
    const bool in_shared = counts_in_shared(n);
    if (in_shared && !allow_shared(reinterpret_cast<const void *>(plan_kernel), 128 * 1024)) return MINW_ECUDA;
    const size_t smem = in_shared ? (size_t)(n + 1) * COUNTS * 4 : 0;
    return launch_pdl(plan_kernel, dim3(1), dim3(PLAN_THREADS), smem, s, ids, T, n, most, p, in_shared ? 1 : 0) == cudaSuccess
               ? MINW_OK : launch_failed();
}

cudaError_t launch_clusters(void (*kern)(Args), const Args &a, int64_t tiles, int smem, int most, cudaStream_t s) {
    if (!allow_shared(reinterpret_cast<const void *>(kern), most)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * a.split));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

template <typename TI, typename TP, int MT, int NT>
static cudaError_t launch_narrow(const Args &a, int64_t tiles, cudaStream_t s) {
    constexpr int bytes = NarrowRing<TI, TP, MT, NT, false>::BYTES, odd = NarrowRing<TI, TP, MT, NT, true>::BYTES;
    return a.in_vec && a.p1_vec ? launch_clusters(narrow_kernel<TI, TP, MT, NT, false>, a, tiles, bytes, bytes, s)
                                : launch_clusters(narrow_kernel<TI, TP, MT, NT, true>, a, tiles, odd, odd, s);
}

template <typename TI, typename TP>
static cudaError_t launch_types(const Args &a, int64_t tiles, cudaStream_t s) {
    return a.r <= 16 ? launch_narrow<TI, TP, 4, 2>(a, tiles, s) : a.r <= 32 ? launch_narrow<TI, TP, 4, 4>(a, tiles, s)
                     : a.most == 32 ? launch_narrow<TI, TP, 2, 8>(a, tiles, s) : launch_narrow<uint16_t, uint16_t, 4, 8>(a, tiles, s);
}

template <typename TP, bool ODD>
static cudaError_t launch_widen_of(const Args &a, int64_t tiles, cudaStream_t s) {
    constexpr int ring = WARPS * (WidenRing<TP, ODD>::DEPTH * WidenRing<TP, ODD>::UNIT + STAGE_BYTES);
    auto kern = a.fine ? widen_kernel<TP, true, ODD> : widen_kernel<TP, false, ODD>;
    if (!allow_shared(reinterpret_cast<const void *>(kern), ring + 3 * 32 * (MAX_RANK + 8) * 2)) return cudaErrorInvalidValue;
    // two blocks an SM, each of eight blocks of columns or more
    const int blocks = (a.E + 63) / 64, sms = num_sms() > 0 ? num_sms() : 152;
    const int64_t groups = std::max<int64_t>(1, std::min<int64_t>((blocks + WARPS - 1) / WARPS, 3 * sms / tiles));
    const int per = (int)((blocks + groups - 1) / groups + WARPS - 1) / WARPS * WARPS, g = (blocks + per - 1) / per;
    return launch_pdl(kern, dim3((unsigned)(tiles * g)), dim3(THREADS), (size_t)ring + (a.fine ? 3 : 2) * a.most * (a.rp + 8) * 2, s, a, g, per);
}

template <typename TP>
static cudaError_t launch_widen(const Args &a, int64_t tiles, cudaStream_t s) {
    return a.p2_vec ? launch_widen_of<TP, false>(a, tiles, s) : launch_widen_of<TP, true>(a, tiles, s);
}

static bool vec_rows(const void *p, int64_t ld, int bf16) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % (bf16 ? 8 : 4) == 0;
}

// One pass through the adapters; types as in the public calls.  plan null: T <= SMALL.
static minw_status through(Args a, int in_bf16, int p_bf16, const Plan *plan, cudaStream_t s) {
    a.rp = rank_pitch(a.r);
    a.in_vec = vec_rows(a.in, a.ld_in, in_bf16);
    a.p1_vec = vec_rows(a.p1, a.D, p_bf16);
    a.p2_vec = vec_rows(a.p2, a.E, p_bf16);
    a.base_vec = vec_rows(a.base, a.ld_base, a.base_bf16);
    a.out_vec = vec_rows(a.out, a.ld_out, a.out_bf16);
    a.scale_vec = vec_rows(a.scale, 4, 0) && vec_rows(a.shift, 4, 0);
    if (plan) a.plan = *plan;
    const int64_t tiles = plan ? tiles_of(a.T, a.n, a.most) : a.T;
    // a block an SM: as many blocks to a tile as there are SMs for
    const int sms = num_sms() > 0 ? num_sms() : 152;
    a.split = 8;
    while (plan && a.split > 1 && tiles * a.split > sms + sms / 8) a.split /= 2;         // (tiles: a bound, mostly above)
    if (!plan) return launch_few(a, in_bf16, p_bf16, s) == cudaSuccess ? launch_status() : launch_failed();
    cudaError_t e = in_bf16 ? (p_bf16 ? launch_types<uint16_t, uint16_t>(a, tiles, s)
                                      : launch_types<uint16_t, float>(a, tiles, s))
                            : (p_bf16 ? launch_types<float, uint16_t>(a, tiles, s)
                                      : launch_types<float, float>(a, tiles, s));
    if (e == cudaSuccess && a.E > 0)
        e = p_bf16 ? launch_widen<uint16_t>(a, tiles, s) : launch_widen<float>(a, tiles, s);
    return e == cudaSuccess ? launch_status() : launch_failed();
}

template <typename TZ, int RT, bool ODD>
static cudaError_t launch_grads_as(const GradArgs &a, int64_t grid, cudaStream_t s) {
    constexpr int bytes = GradRing<TZ, RT, ODD>::ALL;
    if (!allow_shared(reinterpret_cast<const void *>(grads_kernel<TZ, RT, ODD>), bytes)) return cudaErrorInvalidValue;
    return launch_pdl(grads_kernel<TZ, RT, ODD>, dim3((unsigned)grid), dim3(THREADS), bytes, s, a);
}
template <typename TZ, int RT>
static cudaError_t launch_grads_of(const GradArgs &a, int64_t grid, cudaStream_t s) {
    return a.job[0].odd || (a.jobs > 1 && a.job[1].odd) ? launch_grads_as<TZ, RT, true>(a, grid, s) : launch_grads_as<TZ, RT, false>(a, grid, s);
}

template <typename TZ>
static cudaError_t launch_grads(const GradArgs &a, int64_t grid, cudaStream_t s) {
    return a.r <= 16 ? launch_grads_of<TZ, 1>(a, grid, s) : a.r <= 32 ? launch_grads_of<TZ, 2>(a, grid, s) : launch_grads_of<TZ, 4>(a, grid, s);
}

struct Shape {
    int64_t T;
    int K, O, n, r;
};

static bool sizes_fit(const Shape &z) {
    if (z.T >= (1 << 27) || z.K > (1 << 28) || z.O > (1 << 28) || z.r > MAX_RANK || z.n >= (1 << 24)) return false;
    const int64_t tiles = tiles_of(z.T, z.n, rows_of(z.r, false)), blocks = (z.K + 63) / 64 + (z.O + 63) / 64 + 2;
    return z.n * blocks < (1ll << 31) && tiles * std::max<int64_t>(8, blocks) < (1ll << 31);
}

static bool aligned(const void *p, int type) { return reinterpret_cast<uintptr_t>(p) % (type == MINW_BF16 ? 2 : 4) == 0; }
static bool known(int type) { return type == MINW_F32 || type == MINW_BF16; }

}  // namespace adapters
}  // namespace minw

using namespace minw;
using namespace minw_host;

extern "C" {

size_t minw_adapters_workspace_bytes(int64_t T, int32_t K, int32_t O, int32_t n, int32_t r, int32_t backward) {
    using namespace adapters;
    const Shape z{T, K, O, n, r};
    if (T < 0 || K < 1 || O < 1 || n < 1 || r < 1 || !sizes_fit(z)) return 0;
    const int64_t terms = w4_bytes(T, O);
    if (!backward && T <= SMALL) return (size_t)std::max<int64_t>(16, terms);        // no plan (which grows with n)
    int64_t used;
    plan_at(nullptr, T, n, r, &used);
    used += 3 * T * rank_pitch(r) * 2;
    if (backward) return (size_t)(used + 3 * T * rank_pitch(r) * 2);
    return (size_t)std::max<int64_t>(used, terms);
}

minw_status minw_adapters(const void *x, int32_t x_type, int64_t ldx, int64_t T, int32_t K, const int32_t *ids,
                          const void *down, const void *up_, int32_t p_type, int32_t n, int32_t r, const float *alpha,
                          const void *base, int32_t base_type, int64_t ldbase, int32_t O, const float *scale,
                          const float *shift, int32_t act, void *y, int32_t y_type, int64_t ldy, float *h, void *workspace,
                          size_t workspace_bytes, void *stream) {
    using namespace adapters;
    if (T < 0 || K < 1 || O < 1 || n < 1 || r < 1 || ldx < K || ldy < O || (base && ldbase < O)) return MINW_EINVAL;
    if (!down || !up_ || (T > 0 && (!x || !ids || !y)) || act < MINW_ACT_NONE || act > MINW_ACT_SILU) return MINW_EINVAL;
    if (!known(x_type) || !known(p_type) || !known(y_type) || (base && !known(base_type))) return MINW_EINVAL;
    if (!aligned(x, x_type) || !aligned(down, p_type) || !aligned(up_, p_type) || !aligned(y, y_type) ||
        (base && !aligned(base, base_type)) || !on_floats(alpha, scale, shift, h) || !aligned(ids, MINW_F32))
        return MINW_EINVAL;
    if (base && base == y && (base_type != y_type || ldbase != ldy)) return MINW_EINVAL;
    if (x && x == y) return MINW_EINVAL;
    if (!sizes_fit(Shape{T, K, O, n, r})) return MINW_EUNSUPPORTED;
    if (T == 0) return MINW_OK;
    if (!workspace || !aligned16(workspace) || workspace_bytes < minw_adapters_workspace_bytes(T, K, O, n, r, 0)) return MINW_EINVAL;
    Args a{};
    a.in = x; a.ld_in = ldx; a.D = K; a.E = O; a.T = (int)T; a.ids = ids; a.p1 = down; a.p2 = up_; a.n = n; a.r = r;
    a.alpha = alpha; a.base = base; a.base_bf16 = base_type == MINW_BF16; a.ld_base = ldbase; a.scale = scale; a.shift = shift;
    a.act = act; a.out = y; a.out_bf16 = y_type == MINW_BF16; a.ld_out = ldy; a.h = h;
    a.fine = !a.out_bf16 || h;
    a.most = rows_of(r, x_type == MINW_BF16 && p_type == MINW_BF16);
    cudaStream_t s = (cudaStream_t)stream;
    if (T <= SMALL) return through(a, x_type == MINW_BF16, p_type == MINW_BF16, nullptr, s);
    int64_t used;
    const Plan p = plan_at(static_cast<uint8_t *>(workspace), T, n, r, &used);
    a.hp = reinterpret_cast<uint16_t *>(static_cast<uint8_t *>(workspace) + used);
    const minw_status st = make_plan(p, ids, (int)T, n, a.most, s);
    return st != MINW_OK ? st : through(a, x_type == MINW_BF16, p_type == MINW_BF16, &p, s);
}

minw_status minw_w4_adapters(const void *x, int32_t x_type, int64_t ldx, int64_t T, const uint8_t *codes,
                             const uint16_t *scales, int32_t O, int32_t K, int32_t group, const int32_t *ids, const void *down,
                             const void *up_, int32_t p_type, int32_t n, int32_t r, const float *alpha, const float *scale,
                             const float *shift, int32_t act, void *y, int32_t y_type, int64_t ldy, void *workspace,
                             size_t workspace_bytes, void *stream) {
    using namespace adapters;
    if (T < 0 || K < 1 || O < 1 || n < 1 || r < 1 || !down || !up_ || (T > 0 && !ids) || !known(p_type)) return MINW_EINVAL;
    if (!aligned(down, p_type) || !aligned(up_, p_type) || !aligned(ids, MINW_F32) || !on_floats(alpha) || (x && x == y))
        return MINW_EINVAL;
    const minw_status ok = w4::check(x, x_type, ldx, T, codes, scales, O, K, group, scale, shift, act, y, y_type, ldy);
    if (ok != MINW_OK) return ok;
    if (!sizes_fit(Shape{T, K, O, n, r})) return MINW_EUNSUPPORTED;
    if (T == 0) return MINW_OK;
    if (!workspace || !aligned16(workspace) || workspace_bytes < (size_t)w4_bytes(T, O)) return MINW_EINVAL;
    const int xs = x_type == MINW_BF16 ? 2 : 4, ys = y_type == MINW_BF16 ? 2 : 4;
    // the products of so many rows read the weights once (bf16 x); their adapters' terms go through the workspace
    for (int64_t t0 = 0; t0 < T; t0 += W4_ROWS) {
        const int rows = (int)std::min<int64_t>(W4_ROWS, T - t0);
        Args a{};
        a.in = static_cast<const uint8_t *>(x) + t0 * ldx * xs; a.ld_in = ldx; a.D = K; a.E = O; a.T = rows; a.ids = ids + t0;
        a.p1 = down; a.p2 = up_; a.n = n; a.r = r; a.alpha = alpha; a.out = workspace; a.ld_out = O; a.fine = 1;
        const minw_status st = through(a, x_type == MINW_BF16, p_type == MINW_BF16, nullptr, (cudaStream_t)stream);
        if (st != MINW_OK) return st;
        const minw_status sw = w4::matvec(a.in, x_type, ldx, rows, codes, scales, O, K, group, scale, shift, act,
                                          static_cast<uint8_t *>(y) + t0 * ldy * ys, y_type, ldy,
                                          static_cast<const float *>(workspace), (cudaStream_t)stream);
        if (sw != MINW_OK) return sw;
    }
    return MINW_OK;
}

minw_status minw_adapters_backward(const void *x, int32_t x_type, int64_t ldx, int64_t T, int32_t K, const int32_t *ids,
                                   const void *down, const void *up_, int32_t p_type, int32_t n, int32_t r, const float *alpha,
                                   const float *h, const void *dy, int32_t dy_type, int64_t lddy, int32_t O, void *dx,
                                   int64_t lddx, int32_t accumulate, float *ddown, float *dup, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    using namespace adapters;
    if (T < 0 || K < 1 || O < 1 || n < 1 || r < 1 || ldx < K || lddy < O || (dx && lddx < K)) return MINW_EINVAL;
    if (!down || !up_ || (T > 0 && (!ids || !dy || (ddown && !x) || (dup && !h)))) return MINW_EINVAL;
    if (!known(x_type) || !known(p_type) || !known(dy_type)) return MINW_EINVAL;
    if (!aligned(x, x_type) || !aligned(down, p_type) || !aligned(up_, p_type) || !aligned(dy, dy_type) || !aligned(dx, x_type) ||
        !aligned(ids, MINW_F32) || !on_floats(alpha, h, ddown, dup))
        return MINW_EINVAL;
    if (dx && (dx == x || dx == dy)) return MINW_EINVAL;
    if (!sizes_fit(Shape{T, K, O, n, r})) return MINW_EUNSUPPORTED;
    if (!dx && !ddown && !dup) return MINW_OK;
    if (T == 0 && !ddown && !dup) return MINW_OK;
    if (!workspace || !aligned16(workspace) || workspace_bytes < minw_adapters_workspace_bytes(T, K, O, n, r, 1)) return MINW_EINVAL;
    cudaStream_t s = (cudaStream_t)stream;
    int64_t used;
    const Plan p = plan_at(static_cast<uint8_t *>(workspace), T, n, r, &used);
    uint16_t *hp = reinterpret_cast<uint16_t *>(static_cast<uint8_t *>(workspace) + used);
    uint16_t *hh = hp + 3 * T * rank_pitch(r);
    const int most = rows_of(r, dy_type == MINW_BF16 && p_type == MINW_BF16);
    minw_status st = make_plan(p, ids, (int)T, n, most, s);
    if (st != MINW_OK) return st;
    if (T > 0) {
        Args a{};
        a.in = dy; a.ld_in = lddy; a.D = O; a.E = dx ? K : 0; a.T = (int)T; a.ids = ids; a.p1 = up_; a.p2 = down; a.n = n; a.r = r;
        a.alpha = alpha; a.out = dx; a.out_bf16 = x_type == MINW_BF16; a.ld_out = lddx;
        if (accumulate) { a.base = dx; a.base_bf16 = a.out_bf16; a.ld_base = lddx; }
        a.hp = hp;
        a.hh = dup ? hh : nullptr;
        a.h_in = h;
        a.fine = !a.out_bf16 || ddown;
        a.most = most;
        st = through(a, dy_type == MINW_BF16, p_type == MINW_BF16, &p, s);
        if (st != MINW_OK) return st;
    }
    // jobs of one type in one launch
    GradArgs ga{};
    ga.T = (int)T; ga.n = n; ga.r = r; ga.rp = rank_pitch(r); ga.plan = p; ga.beside = dx && T > 0;
    // Warps share a user's rows while the blocks that this makes are four for an SM, if each keeps a step of 16 rows.  Beside dx,
    // whose blocks hold half of the SMs' places, a third and a fourth block only if each warp keeps 64 rows: users of 341 rows at
    // 4096 + 4096 columns take 57 us, left at two blocks 68; users of 50 rows at 3001 + 2777 columns take 61 us (fp32) and 41
    // (bf16), shared 70 and 47; without dx shared 44 and 31, left at two blocks 56 and 36.
    const int sms = num_sms() > 0 ? num_sms() : 152;
    const int64_t columns = ((ddown ? (K + 63) / 64 : 0) + (dup ? (O + 63) / 64 : 0)) * (int64_t)n;
    ga.along = 1;
    while (ga.along < WARPS / 2 && columns * ga.along / WARPS <= 2 * sms &&
           T / n >= (ga.beside && columns * 2 * ga.along / WARPS > 2 * sms ? 64 : 16) * ga.along)
        ga.along *= 2;
    const int wide = 64 * (WARPS / ga.along);
    const Job jobs[2] = {{hp, x, ddown, ldx, K, (K + wide - 1) / wide, !vec_rows(x, ldx, x_type == MINW_BF16), vec_rows(ddown, K, 0)},
                         {hh, dy, dup, lddy, O, (O + wide - 1) / wide, !vec_rows(dy, lddy, dy_type == MINW_BF16), vec_rows(dup, O, 0)}};
    const int types[2] = {x_type, dy_type};
    for (int k = 0; k < 2; ++k) {
        if (!jobs[k].out) continue;
        ga.job[0] = jobs[k];
        ga.jobs = 1;
        int64_t grid = (int64_t)n * jobs[k].blocks;
        if (k == 0 && jobs[1].out && types[0] == types[1]) {
            ga.job[1] = jobs[1];
            ga.jobs = 2;
            grid += (int64_t)n * jobs[1].blocks;
            ++k;
        }
        const cudaError_t e = types[k] == MINW_BF16 ? launch_grads<uint16_t>(ga, grid, s) : launch_grads<float>(ga, grid, s);
        if (e != cudaSuccess) return launch_failed();
    }
    return launch_status();
}

}  // extern "C"
