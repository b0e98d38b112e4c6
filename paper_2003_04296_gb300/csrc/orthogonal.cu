// orthogonal.cu -- orthogonalised updates of lists of matrices: each matrix divided
// by its norm and taken through Newton-Schulz products, which bring its singular
// values to about 1.
//
// One step is X <- (a I + b A + c A^2) X with A = X X^T of the smaller side, m x m.
// Every step is a polynomial in the first A times X, and polynomials in A commute
// and are symmetric, so several steps (a stage) run on m x m matrices alone:
//   Z = a I + b A + c A^2,   Q <- Z Q,   A <- (Z A) Z
// and Q X comes once at the stage's end: for n >= m a third of the direct form's
// operations, half of them on symmetric results whose other half is a mirror image.
// What that costs is precision: an error e of A counts 11.9^steps e where the singular
// values are small, and Q is up to 41 times what it leaves of strong directions.  So
// - every matrix is held as the sum of two fp16 numbers (22 bits), and a product takes
//   three fp16 products, lo hi + hi lo + hi hi;
// - the tensor cores cut each addend at 2^-25 of the largest and what they add to, so they
//   sum up 32 of K (pairs of blocks 64), and fp32 registers the rest, to nearest;
// - Z and Q are held without their identity parts, Z = a I + W and Q = q I + R with q = a^steps:
//     W = b A + c A^2,   Z A = a A + W A,   R <- q W + a R + W R,   Q X = q X + R X,
//   and what the identity contributes is added in fp32, outside the truncated sums;
// - all tiles of a matrix read a block of the diagonal the same way, else its roundings, which are
//   not symmetric, do not cancel (600 x 700 of noise 7e-6 off instead of 2.5e-6);
// - a stage has three steps at most (five: 3e-3 to 9e-3).
// Against the formula in 64 bits (Frobenius; plain fp32 products in parentheses), noise / a gradient of few strong
// directions: 128 x 1152 1.8e-6 / 1.8e-6 (1.2e-6 / 1.2e-6), 1024 x 8192 2.6e-6 / 1.2e-6 (3.9e-6 / 3.5e-6),
// 4096 x 4096 2.2e-6 / 1.4e-6 (4.8e-6 / 6.6e-6).  Without all this but the stages, sums of 128 of K:
// 8.7e-6 / 1.0e-5, 7.1e-6 / 5.4e-6 and 6.0e-6 / 5.0e-6, at 116 us instead of 126, 318 instead of 336,
// 2.77 ms instead of 2.89.
//
// The scales are powers of two that the mathematics gives: a matrix of Frobenius norm
// f in [1/2, 1) 2^e enters as X 2^(15 - e), so that nothing overflows and the smallest
// part lost is 2^-40 of the norm; singular values stay below 1.2025 from then on,
// A below 1.447, W below 2.81, R below 3.4446^steps.
//
// Operands lie in the workspace as the tensor cores read them: blocks of 128 rows x 64
// columns, 16 KB, swizzled in rows of 128 bytes.  Such a block is a K-major operand of
// 128 rows or, column group by column group, an MN-major one, so X serves X X^T, X^T X, Q X and
// X Q without a transposed copy, a symmetric matrix is its lower triangle alone, blocks travel
// as plain bulk copies, and no matrix of a list needs a tensor map.
//
// A list goes through the kernels together: level k of all its matrices is one launch.
// What bounds a level: where tiles are many, the way from L2 into the SMs (64 bytes a clock: 64 KB
// for 64 of K, 0.55 to 0.67 us a tile of 128 x 128, of which the tensor cores need 0.4), so
// pairs of blocks take 256 x 256; where they are few, latency (2.5 us between two launches, 4.5 for a
// tile's start and end), so clusters split K.  4096 x 4096 of bf16 2.8 to 2.9 ms (1.4 of the 1.88
// PFLOP/s that a library's bf16 product reaches), 1024 x 8192 of fp32 336 us, 128 x 1152 126, 10 x 1024 11.
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "kernels.cuh"
#include "split.cuh"
#include "values.cuh"

namespace cg = cooperative_groups;

namespace minw {

static __device__ int g_orth_error = 0;

namespace orth {

constexpr int T = 128;                       // rows and columns of a tile
constexpr uint32_t BLOCK = 16384;            // bytes of 128 rows x 64 columns of fp16
constexpr int THREADS = 256;
constexpr int LOADER = 8, ISSUER = 9;        // a product's warps beside the eight that take its sums
constexpr int STAGES = 3;
constexpr uint32_t STAGE = 4 * BLOCK;        // hi and lo of both operands, 64 of K
constexpr int EARLY = 4;                     // steps of a tile's end, 16 rows each, whose added values are ready before the sums are
constexpr int PITCH = 132;                   // floats between rows of a tile in shared memory
constexpr int CAP = 224;                     // matrices of a launch
constexpr int FEW = 16;                      // ... of a launch with short arguments
constexpr float CA = 3.4445f, CB = -4.7750f, CC = 2.0315f;
constexpr int SLOTS = 6;                     // m x m matrices: two for A, Z, Z A, two for Q

struct Stat {
    float scale1, scale2;                    // X = these two times the matrix
    float gram;                              // 1 / mu^2, with mu the norm of X 2^-15
    float apply;                             // 1 / mu
    int finite;
};

// Levels on m x m results: Gram matrices, one product, two at a time.
enum Kind { OF_X, ONE, TWO };

struct Mat {
    const void *g;
    float *mom;
    void *out;
    uint8_t *x0, *x1, *small;                // hi blocks, then lo blocks; `small`: SLOTS of them
    int64_t ldg, ldm, ldo;
    int rows, cols;
    int full0;                               // tiles of X of the matrices before
    int pair_tri0, pair_full0;               // ... clusters for pairs
    int first[3], split[3];                  // of each Kind: clusters of the matrices before; shares of K of a tile
    float limit, rate;
    uint8_t g_bf16, o_bf16, tall, gvec, mvec, ovec;

    __host__ __device__ int rb() const { return (rows + T - 1) / T; }
    __host__ __device__ int cb() const { return (cols + T - 1) / T; }                   // of 128 columns
    __host__ __device__ int mb() const { return tall ? cb() : rb(); }
    __host__ __device__ int side() const { return tall ? cols : rows; }
};

struct Sizes {
    int count, full;                         // matrices; tiles of X
    int pair_tri, pair_full;                 // clusters for pairs, four tiles each: of lower triangles, of X
    bool pairs, pairs_x;                     // blocks work in pairs: in the levels on m x m results, in those on X
    int clusters[3], blocks[3];              // of each Kind, for one product: clusters, their blocks
    const Mat *table;                        // in the workspace
    Stat *stat;
    double *part;                            // a sum of squares for each tile of X
};

template <int N>
struct Table {
    Mat m[N];
};
static_assert(sizeof(Table<CAP>) + sizeof(Sizes) + 16 <= 32764, "a launch's arguments");
template <>
struct Table<0> {
    Mat *m = nullptr;
};

// The matrix of tile or cluster t: the last one that begins at or before it.
template <typename F>
__device__ __forceinline__ int find(int count, int t, F first) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first(mid) <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Byte of (row, column) in a block.
__device__ __forceinline__ uint32_t at(int r, int c) {
    return (uint32_t)(r * 128 + ((((c >> 3) ^ r) & 7) << 4) + (c & 7) * 2);
}

// v as the sum of two fp16 numbers, eight values: one 16-byte store each.
__device__ __forceinline__ void split8(const float *v, uint4 &hi, uint4 &lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __half2 a = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
        const float2 f = __half22float2(a);
        const __half2 b = __floats2half2_rn(v[2 * k] - f.x, v[2 * k + 1] - f.y);
        h[k] = *reinterpret_cast<const uint32_t *>(&a);
        l[k] = *reinterpret_cast<const uint32_t *>(&b);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}

__device__ __forceinline__ void join8(const uint4 &hi, const uint4 &lo, float *v) {
    const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&h[k]));
        const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&l[k]));
        v[2 * k] = a.x + b.x;
        v[2 * k + 1] = a.y + b.y;
    }
}

// ---------------------------------------------------------------------------
// The matrix in: its norm, then its scaled blocks and the momentum's step
// ---------------------------------------------------------------------------

struct Step {
    float mu;
    int use, nesterov;                       // use: a momentum is given
};

template <typename V>
__device__ __forceinline__ void load8(const V *p, int64_t at_, int left, bool vec, float *v) {
    if (vec && left >= 8) {
        Vec<V, 8> w;
        w.load(p + at_);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = w.get(i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.0f;
            if (i < left) {
                Vec<V, 1> w;
                w.load(p + at_ + i);
                v[i] = w.get(0);
            }
        }
    }
}

template <typename V>
__device__ __forceinline__ void store8(V *p, int64_t at_, int left, bool vec, const float *v) {
    if (vec && left >= 8) {
        Vec<V, 8> w;
        w.set(v);
        w.store(p + at_);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) {
                Vec<V, 1> w;
                w.set(v + i);
                w.store(p + at_ + i);
            }
    }
}

// Eight values of row r from column c on: the momentum's step m = mu m + g and what is orthogonalised, u.  Zeros outside.
__device__ __forceinline__ void value8(const Mat &m, const Step &s, int r, int c, float *u, float *mom) {
    const int left = r < m.rows ? m.cols - c : 0;
    if (m.g_bf16) load8(static_cast<const uint16_t *>(m.g), r * m.ldg + c, left, m.gvec, u);
    else load8(static_cast<const float *>(m.g), r * m.ldg + c, left, m.gvec, u);
    if (s.use) {
        load8(m.mom, r * m.ldm + c, left, m.mvec, mom);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            mom[i] = fmaf(s.mu, mom[i], u[i]);
            u[i] = s.nesterov ? fmaf(s.mu, mom[i], u[i]) : mom[i];
        }
    }
}

__device__ __forceinline__ double sum64(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// A block's tile: 128 rows x 128 columns, eight values a thread at a time.
template <int N>
__global__ void __launch_bounds__(THREADS) squares_kernel(const __grid_constant__ Table<N> table, Sizes l, Step s) {
    pdl_wait();
    pdl_trigger();
    __shared__ double red[THREADS / 32];
    // the list's matrices into the workspace, where the kernels after this one find them (a launch with all of
    // a long list in its arguments takes the host three times as long)
    if (blockIdx.x == 0) {
        static_assert(sizeof(Mat) % 8 == 0, "whole words");
        const uint64_t *from = reinterpret_cast<const uint64_t *>(&table);
        uint64_t *to = reinterpret_cast<uint64_t *>(const_cast<Mat *>(l.table));
        for (int k = threadIdx.x; k < l.count * (int)(sizeof(Mat) / 8); k += THREADS) to[k] = from[k];
    }
    const Mat &m = table.m[find(l.count, blockIdx.x, [&](int k) { return table.m[k].full0; })];
    const int t = blockIdx.x - m.full0, r0 = t / m.cb() * T + (threadIdx.x >> 4), c = t % m.cb() * T + (threadIdx.x & 15) * 8;
    float sum = 0.0f;
    double d = 0.0;
#pragma unroll 2
    for (int k = 0; k < T; k += 16) {
        float u[8], mom[8], q = 0.0f;
        bool some = false;
        value8(m, s, r0 + k, c, u, mom);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            q = fmaf(u[i], u[i], q);
            some = some || u[i] != 0.0f;
        }
        // squares that leave fp32's range (or may have lost bits to it) are added in fp64
        if (q >= 1e-30f && q <= 1e35f) sum += q;
        else if (some)
#pragma unroll 1
            for (int i = 0; i < 8; ++i) d = fma((double)u[i], (double)u[i], d);
    }
    d = sum64(d + (double)sum);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = d;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < THREADS / 32; ++k) d += red[k];
        l.part[blockIdx.x] = d;
    }
}

__global__ void __launch_bounds__(THREADS) enter_kernel(Sizes l, Step s, int lo_part) {
    pdl_wait();
    pdl_trigger();
    __shared__ double red[THREADS / 32];
    __shared__ Stat st;
    const int which = find(l.count, blockIdx.x, [&](int k) { return l.table[k].full0; });
    const Mat m = l.table[which];
    const int t = blockIdx.x - m.full0, tiles = m.rb() * m.cb();
    double d = 0.0;
    for (int k = threadIdx.x; k < tiles; k += THREADS) d += l.part[m.full0 + k];
    d = sum64(d);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = d;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < THREADS / 32; ++k) d += red[k];
        int e = 0;
        const bool finite = d <= 1.7e308;
        const double mu = finite && d > 0.0 ? frexp(sqrt(d), &e) : 1.0;        // the norm is mu 2^e
        st.finite = finite;
        // 2^(15 - e) in two factors, each an fp32 number for every e from -149 to 150
        const int h = (15 - e) / 2;
        st.scale1 = finite ? ldexpf(1.0f, h) : 0.0f;
        st.scale2 = finite ? ldexpf(1.0f, 15 - e - h) : 0.0f;
        st.apply = (float)(1.0 / mu);
        st.gram = (float)(1.0 / (mu * mu));
        if (t == 0) l.stat[which] = st;
    }
    __syncthreads();
    const int rt = t / m.cb(), ct = t % m.cb(), c8 = (threadIdx.x & 15) * 8, c = ct * T + c8;
    const int64_t blocks = (int64_t)m.rb() * m.cb() * 2;
    uint8_t *b = m.x0 + ((int64_t)rt * m.cb() * 2 + ct * 2 + (c8 >> 6)) * BLOCK;
#pragma unroll 2
    for (int k = threadIdx.x >> 4; k < T; k += 16) {
        float u[8], mom[8];
        const int r = rt * T + k;
        value8(m, s, r, c, u, mom);
        if (s.use && st.finite && r < m.rows) store8(m.mom, r * m.ldm + c, m.cols - c, m.mvec, mom);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = st.finite ? u[i] * st.scale1 * st.scale2 : 0.0f;
        uint4 hi, lo;
        split8(u, hi, lo);
        *reinterpret_cast<uint4 *>(b + at(k, c8 & 63)) = hi;
        if (lo_part) *reinterpret_cast<uint4 *>(b + blocks * BLOCK + at(k, c8 & 63)) = lo;
    }
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------

__device__ __forceinline__ float clipped(float w, float rate, float z, float limit) {
    const float n = fmaf(rate, z, w);
    return n > limit ? limit : n < -limit ? -limit : n;
}

enum Mode { GRAM, MUL, APPLY, LEAVE };

struct Product {
    int p, q, out;                           // slots of the factors and the result (LEAVE, APPLY: p = R)
    float factor;                            // of the sum, on its way to the result's scale
    int add[2];                              // slots of what is added to it, -1: none (LEAVE, APPLY: X) ...
    float times[2];                          // ... so many times
};

struct Level {
    int mode, products, split;               // split: blocks of a cluster
    int upper;                               // the m x m matrices were made by pairs
    Product pr[2];
    int later;                               // GRAM, APPLY, LEAVE: of a later stage than the first
    int x1;                                  // ... X is in x1 (every other stage; APPLY writes the other one)
    int x_lo;                                // ... and has a lo part
    int update;                              // LEAVE: weights are updated
    float lr;
    long long wait_cycles;
};

__device__ __forceinline__ uint32_t su32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t *b, uint32_t n) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(su32(b)), "r"(n));
}
__device__ __forceinline__ bool bar_try(uint64_t *b, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(su32(b)), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool bar_wait(uint64_t *b, uint32_t parity, long long limit) {
    if (bar_try(b, parity)) return true;
    const long long t0 = clock64();
    while (!bar_try(b, parity)) {
        if (clock64() - t0 > limit) {
            atomicExch(&g_orth_error, 1);
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }

// Blocks in shared memory.  K-major: rows of 64 K values, eight rows 1024 bytes on.  MN-major: pieces of 64 columns, 64
// rows of K each (8 KB), eight rows of K 1024 bytes on.
__device__ __forceinline__ uint64_t desc(uint32_t addr, bool mn) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(mn ? 8192u >> 4 : 1u) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// (By one thread, as are the commits.)
__device__ __forceinline__ bool elected() {
    uint32_t e;
    asm volatile("{\n .reg .pred p;\n .reg .b32 r;\n elect.sync r|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(e));
    return e != 0;
}
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}
__device__ __forceinline__ void mma_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(su32(bar)) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const uint8_t *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(su32(bar))
                 : "memory");
}

// An operand of a tile: hi blocks at `p`, lo blocks `lo` bytes on (0: none), `wide` blocks to a row of blocks.  A symmetric
// matrix is held as its lower triangle of tiles: a block of the upper one is the mirror image's, read the other way.
struct Side {
    const uint8_t *p;
    int64_t lo;
    int wide, tile;
    bool mn, sym;
    // PAIR: tiles 2 p and 2 p + 1 are read the same way, from 2 p + 2 on as mirror images; levels of pairs leave tile (2 p, 2 p + 1) for
    // that.  Without it (APPLY and LEAVE after levels without pairs) from 2 p + 1 on: a block on the diagonal is its mirror image then.
    // (So in all levels, its own roundings count: 600 x 700 of noise 7e-6 off instead of 2.4e-6.)
    int last = -1;                           // the last tile that is read as it lies, -1: `tile`

    __device__ __forceinline__ bool turned(int kb) const { return sym ? (kb >> 1) > (last < 0 ? tile : last) : mn; }
    __device__ __forceinline__ void load(uint32_t dst, int kb, uint64_t *bar) const {
        if (!turned(kb)) {
            const uint8_t *s = p + ((int64_t)tile * wide + kb) * BLOCK;
            bulk_load(dst, s, BLOCK, bar);
            if (lo) bulk_load(dst + BLOCK, s + lo, BLOCK, bar);
        } else {
            const uint8_t *s = p + ((int64_t)(kb >> 1) * wide + 2 * tile) * BLOCK + (kb & 1) * (BLOCK / 2);
            bulk_load(dst, s, BLOCK / 2, bar);
            bulk_load(dst + BLOCK / 2, s + BLOCK, BLOCK / 2, bar);
            if (lo) {
                bulk_load(dst + BLOCK, s + lo, BLOCK / 2, bar);
                bulk_load(dst + BLOCK + BLOCK / 2, s + lo + BLOCK, BLOCK / 2, bar);
            }
        }
    }
    __device__ __forceinline__ uint32_t bytes() const { return lo ? 2 * BLOCK : BLOCK; }
};

struct Smem {
    uint64_t full[STAGES], empty[STAGES], peer[STAGES], sums[4], taken[4];
    uint32_t tmem;
};

// Pairs: the even block of a cluster of two issues products of 256 rows for both, each block's rows from its own shared memory, half
// of the second operand from each.
__device__ __forceinline__ void mma_f16_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}
__device__ __forceinline__ void mma_commit_pair(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n" ::"r"(su32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}
// An arrival at the even block's barrier.  RELAXED: of sums read from tensor memory, which the fence before orders; a release waits for
// this thread's other memory operations as well.
template <bool RELAXED>
__device__ __forceinline__ void arrive_even(uint64_t *bar) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;\n" : "=r"(at) : "r"(su32(bar)));
    if constexpr (RELAXED) asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(at) : "memory");
    else asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(at) : "memory");
}

__device__ __forceinline__ void load32(uint32_t addr, uint32_t *w) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, "
        "%13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, "
        "[%32];\n"
        : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]),
          "=r"(w[8]), "=r"(w[9]), "=r"(w[10]), "=r"(w[11]), "=r"(w[12]), "=r"(w[13]), "=r"(w[14]),
          "=r"(w[15]), "=r"(w[16]), "=r"(w[17]), "=r"(w[18]), "=r"(w[19]), "=r"(w[20]), "=r"(w[21]),
          "=r"(w[22]), "=r"(w[23]), "=r"(w[24]), "=r"(w[25]), "=r"(w[26]), "=r"(w[27]), "=r"(w[28]),
          "=r"(w[29]), "=r"(w[30]), "=r"(w[31])
        : "r"(addr));
}
// sum += 64 columns, two an instruction.
__device__ __forceinline__ void add64(uint32_t addr, Pair *sum) {
    uint32_t w[64];
    load32(addr, w);
    load32(addr + 32, w + 32);
    asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
    // (what was loaded is there from here on alone)
#pragma unroll
    for (int k = 0; k < 64; ++k) asm volatile("" : "+r"(w[k]));
#pragma unroll
    for (int k = 0; k < 32; ++k) sum[k] = add2(sum[k], pair(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1])));
}

// PAIR: four tiles by a cluster of two blocks, 256 x 256 sums, whose products read 64 KB a block for 64 of K where four blocks
// by themselves read as much each: it is the way from L2 that products wait for.  Two sums of 256 columns fill the tensor memory;
// registers take them over after 64 of K: 4096 x 4096 in 2.89 ms, after 32 1.03 times that, after 128 0.99 times at 1.4 times the error (noise).
// A tile for itself has four sums of 128 columns, each of 32 of K: 512 x 512 in 186 us (a value at a time instead of two 192); of
// 64 in 0.92 times that at 1.15 times the error, wide matrices of noise at 1.5 to 1.7 times it.
// N: matrices whose descriptions come with the launch, so that a block knows its work before it waits for the kernel before; 0:
// they are read from the workspace, after that wait (what an earlier kernel wrote is there for certain only then).
template <bool PAIR, int N>
__global__ void __launch_bounds__(THREADS + 64, 1) product_kernel(const __grid_constant__ Sizes l, const __grid_constant__ Level v,
                                                                  const __grid_constant__ Table<N> own) {
    constexpr int WIDTH = PAIR ? 2 * T : T;          // columns of a block's tile
    constexpr int MINE = PAIR ? 128 : 64;                       // ... of a thread
    constexpr int SUMS = 512 / WIDTH;                           // sums in tensor memory
    constexpr int SPAN = PAIR ? 64 : 32;                        // of K that the tensor cores sum by themselves
    constexpr int ADDED = PAIR ? 3 : 4;                         // steps of the end whose values are on their way at a time
    static_assert((PAIR ? 2 * T * PITCH * 4 : (STAGES - 1) * STAGE) + ADDED * 4 * THREADS * 16 <= STAGES * STAGE, "in the ring");
    static_assert(STAGES == 3 && T * PITCH * 4 <= (STAGES - 1) * STAGE, "behind the sums");
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *ring = smem_raw + ((1024u - (su32(smem_raw) & 1023u)) & 1023u);
    float *acc = reinterpret_cast<float *>(ring);               // the tile, once the ring is done with
    __shared__ Smem sm;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            bar_init(&sm.full[s], 1);
            bar_init(&sm.empty[s], 1);
            bar_init(&sm.peer[s], 1);
        }
        for (int k = 0; k < SUMS; ++k) {
            bar_init(&sm.sums[k], 1);
            bar_init(&sm.taken[k], (PAIR ? 2 : 1) * THREADS / 32);
        }
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    cg::cluster_group cluster = cg::this_cluster();
    if (warp == ISSUER) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(su32(&sm.tmem)));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(su32(&sm.tmem)));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n");
        }
    }
    fence_before();
    if (PAIR) cluster.sync();                                   // the other block's barriers and columns are there
    else __syncthreads();
    fence_after();
    const uint32_t tmem = sm.tmem;
    if (N == 0) pdl_wait();
    const Mat *table = N == 0 ? l.table : own.m;

    // What this block computes: matrix, product, tile (i, j), share of K.  A cluster takes `split` blocks' work of one
    // matrix: a tile in so many shares, or two tiles in half as many, or ...
    const int split = v.split, in_cluster = blockIdx.x % split, tri = v.mode <= MUL;
    int t = blockIdx.x / split, which = 0;
    const int kind = v.mode == GRAM ? OF_X : v.products == 1 ? ONE : TWO, all = PAIR ? (tri ? l.pair_tri : l.pair_full) : tri ? l.clusters[kind] : l.full;
    if (tri) {
        which = t / all;
        t -= which * all;
    }
    const int index = PAIR  ? find(l.count, t, [&](int k) { return tri ? table[k].pair_tri0 : table[k].pair_full0; })
                      : tri ? find(l.count, t, [&](int k) { return table[k].first[kind]; })
                            : find(l.count, t, [&](int k) { return table[k].full0; });
    const Mat m = table[index];
    const Product pr = v.pr[which];
    const int shares = tri && !PAIR ? table[index].split[kind] : 1, rank = PAIR ? 0 : in_cluster % shares;
    if (PAIR) t -= tri ? m.pair_tri0 : m.pair_full0;
    else t = (t - (tri ? table[index].first[kind] : m.full0)) * (split / shares) + in_cluster / shares;
    bool idle = !PAIR && t >= (tri ? m.mb() * (m.mb() + 1) / 2 : m.rb() * m.cb());     // of a matrix's last cluster
    const int mb = m.mb();
    const int64_t small_blocks = (int64_t)mb * mb * 2 * BLOCK, slot = 2 * small_blocks;
    const int64_t x_blocks = (int64_t)m.rb() * m.cb() * 2 * BLOCK;
    uint8_t *x = v.x1 ? m.x1 : m.x0;
    int i, j;
    bool mute = false;                                          // computed for the other block's sake
    const int columns = tri ? mb : m.cb();                      // of tiles
    if (PAIR) {                                                 // rows 2 p and 2 p + 1, columns 2 q and 2 q + 1
        int p = t / ((m.cb() + 1) / 2), q = t % ((m.cb() + 1) / 2);
        if (tri) {
            p = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
            while ((p + 1) * (p + 2) / 2 <= t) ++p;
            while (p * (p + 1) / 2 > t) --p;
            q = t - p * (p + 1) / 2;
        }
        i = 2 * p + in_cluster;
        j = 2 * q;
        mute = i >= (tri ? mb : m.rb());
    } else if (tri) {
        i = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while ((i + 1) * (i + 2) / 2 <= t) ++i;
        while (i * (i + 1) / 2 > t) --i;
        j = t - i * (i + 1) / 2;
    } else {
        i = t / m.cb();
        j = t % m.cb();
    }
    if (mute) i = min(i, (tri ? mb : m.rb()) - 1);
    const Side sx{x, v.x_lo ? x_blocks : 0, 2 * m.cb(), 0, false, false};
    Side a, b;
    int kbs;                                                    // blocks of 64 along K
    if (v.mode == GRAM) {
        a = b = sx;
        a.tile = i;
        b.tile = j;
        a.mn = b.mn = m.tall;
        kbs = 2 * (m.tall ? m.rb() : m.cb());
    } else {
        const Side sp{m.small + pr.p * slot, small_blocks, 2 * mb, i, false, true};
        const Side sq{m.small + pr.q * slot, small_blocks, 2 * mb, j, false, true};
        kbs = 2 * mb;
        a = sp;
        b = sq;
        if (!tri) {
            if (m.tall) {                                       // X Q
                a = sx;
                a.tile = i;
                b = sp;
                b.tile = j;
            } else {                                            // Q X
                b = sx;
                b.tile = j;
                b.mn = true;
            }
        }
    }
    if (PAIR) {
        b.tile = min(j + in_cluster, columns - 1);
        a.last = v.upper ? a.tile | 1 : a.tile & ~1;
        b.last = v.upper ? b.tile | 1 : b.tile & ~1;
    }
    const int kb0 = idle ? 0 : rank * kbs / shares, kb1 = idle ? 0 : (rank + 1) * kbs / shares;
    const bool same = !PAIR && a.p == b.p && a.tile == b.tile && a.mn == b.mn && a.sym == b.sym;
    const uint32_t bytes = a.bytes() + (same ? 0 : b.bytes());
    if (N > 0) pdl_wait();
    pdl_trigger();
    if (v.mode == LEAVE && v.update && warp < THREADS / 32) {   // weights on their way to L2 during the products: a line a thread
        const int each = m.o_bf16 ? 64 : 32, lines = WIDTH / each;
        for (int e = threadIdx.x; e < T * lines; e += THREADS) {
            const int r = i * T + e / lines, c = j * T + e % lines * each;
            if (r < m.rows && c < m.cols)
                asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint8_t *>(m.out) + (r * m.ldo + c) * (m.o_bf16 ? 2 : 4)));
        }
    }
    // what is added to the sums: values of two slots, or of X
    const Stat st = v.mode != MUL ? l.stat[index] : Stat{};
    const int wide = tri ? 2 * mb : 2 * m.cb(), rows = T / shares, r0 = rank * rows, c = (threadIdx.x & 15) * 8;
    const int64_t lo = tri ? small_blocks : x_blocks;
    // ... 16 rows of this block's share of a tile at a time, eight columns a thread
    const int steps = mute || idle || warp >= THREADS / 32 ? 0 : PAIR && j + 1 < columns ? T / 8 : rows / 16;
    auto row_of = [&](int step) { return r0 + (PAIR ? step % (T / 16) : step) * 16 + (int)(threadIdx.x >> 4); };
    auto tile_of = [&](int step) { return PAIR ? j + step / (T / 16) : j; };
    auto place = [&](int step) {
        return ((int64_t)i * wide + 2 * tile_of(step) + (c >> 6)) * BLOCK + at(row_of(step), c & 63);
    };
    const uint8_t *from[2] = {nullptr, nullptr};
    int64_t from_lo = small_blocks;
    float times[2] = {pr.times[0], pr.times[1]};
    if (v.mode == MUL) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (pr.add[e] >= 0) from[e] = m.small + pr.add[e] * slot;
    } else if (!tri) {
        from[0] = x;
        from_lo = v.x_lo ? x_blocks : 0;
        if (!v.later) times[0] *= st.apply;
    }
    // eight values of them, as their parts lie at w
    auto sum_of = [&](const uint4 (*w)[2], float *f) {
        join8(w[0][0], w[0][1], f);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] *= times[0];
        if (from[1]) {
            float g[8];
            join8(w[1][0], w[1][1], g);
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = fmaf(times[1], g[k], f[k]);
        }
    };
    // The first steps' while the tensor cores are busy, into shared memory behind the ring (all of them at the end, as they were loaded: 2 us
    // of a level's 10); a thread reads back its own.
    float4 *early = reinterpret_cast<float4 *>(ring + STAGES * STAGE) + threadIdx.x;
    if (from[0]) {
#pragma unroll 2
        for (int step = 0; step < min(steps, EARLY); ++step) {
            uint4 w[2][2] = {};
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (from[e]) {
                    w[e][0] = *reinterpret_cast<const uint4 *>(from[e] + place(step));
                    if (from_lo) w[e][1] = *reinterpret_cast<const uint4 *>(from[e] + place(step) + from_lo);
                }
            float f[8];
            sum_of(w, f);
            early[2 * step * THREADS] = make_float4(f[0], f[1], f[2], f[3]);
            early[(2 * step + 1) * THREADS] = make_float4(f[4], f[5], f[6], f[7]);
        }
    }
    // The later steps' as they lie, on their way to shared memory behind the sums.  That is the ring's last stage (of pairs: part of
    // it), which the third last block of K leaves for good, for the stages are taken so.
    const int off = PAIR ? 0 : 2 - (kb1 - kb0) % 3;
    auto stage = [&](int s) { return (uint32_t)((s + off) % STAGES) * STAGE; };
    uint8_t *added = ring + (PAIR ? 2 * T * PITCH * 4 : (STAGES - 1) * (int)STAGE) + threadIdx.x * 16;
    auto fetch = [&](int step) {
        if (step < steps) {
            uint8_t *d = added + step % ADDED * (4 * THREADS * 16);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (from[e]) {
                    copy_async<16>(d + 2 * e * THREADS * 16, from[e] + place(step));
                    if (from_lo) copy_async<16>(d + (2 * e + 1) * THREADS * 16, from[e] + place(step) + from_lo);
                }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto fetch_later = [&]() {
        if (steps > EARLY && from[0])
#pragma unroll 1
            for (int step = EARLY; step < EARLY + ADDED; ++step) fetch(step);
    };
    bool ok = true;
    if (warp == LOADER) {
        if (lane == 0) {
            int s = 0, lap = 0, g = 0;
            for (int kb = kb0; kb < kb1; ++kb, ++g) {
                if (lap > 0 && !bar_wait(&sm.empty[s], (lap - 1) & 1, v.wait_cycles)) break;
                const uint32_t dst = su32(ring) + stage(s);
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(su32(&sm.full[s])),
                             "r"(bytes)
                             : "memory");
                a.load(dst, kb, &sm.full[s]);
                if (!same) b.load(dst + 2 * BLOCK, kb, &sm.full[s]);
                if (++s == STAGES) { s = 0; ++lap; }
            }
            // every load has landed before the ring is used again
            for (int k = g > STAGES ? g - STAGES : 0; k < g; ++k)
                if (!bar_wait(&sm.full[k % STAGES], (k / STAGES) & 1, v.wait_cycles)) break;
        }
        __syncwarp();
    } else if (PAIR && warp == ISSUER && in_cluster == 1) {     // tells the even block what has landed here
        int s = 0;
        uint32_t phase = 0u;
        for (int kb = kb0; kb < kb1 && ok; ++kb) {
            ok = __all_sync(0xffffffffu, bar_wait(&sm.full[s], phase, v.wait_cycles));
            if (ok && lane == 0) arrive_even<false>(&sm.peer[s]);
            if (++s == STAGES) { s = 0; phase ^= 1u; }
        }
    } else if (warp == ISSUER) {
        // D fp32, A and B fp16; bits 15 and 16: MN-major
        int s = 0, sum = 0;
        uint32_t phase = 0u;
        const bool leader = elected();
        for (int kb = kb0; kb < kb1; ++kb) {
            ok = bar_wait(&sm.full[s], phase, v.wait_cycles);
            if (PAIR) ok = ok && bar_wait(&sm.peer[s], phase, v.wait_cycles);
            const uint32_t base = su32(ring) + stage(s);
            const bool at = a.turned(kb), bt = b.turned(kb);
            const uint32_t idesc = (1u << 4) | ((at ? 1u : 0u) << 15) | ((bt ? 1u : 0u) << 16) | ((uint32_t)(WIDTH >> 3) << 17) | ((PAIR ? 16u : 8u) << 24);
            const uint32_t ka = at ? 2048 >> 4 : 32 >> 4, kbk = bt ? 2048 >> 4 : 32 >> 4;      // 16 of K
            const uint64_t ad = desc(base, at), bd = desc(same ? base : base + 2 * BLOCK, bt);
#pragma unroll
            for (int half = 0; half < 64 / SPAN; ++half, ++sum) {
                if (sum >= SUMS) ok = ok && bar_wait(&sm.taken[sum % SUMS], (sum / SUMS - 1) & 1, v.wait_cycles);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                fence_after();
                if (leader) {
                    const uint32_t d = WIDTH * (sum % SUMS);    // (all columns are this block's: they begin at 0)
                    uint32_t on = 0u;
                    auto add = [&](uint64_t x_, uint64_t y_) {
#pragma unroll
                        for (int k = half * SPAN / 16; k < (half + 1) * SPAN / 16; ++k) {
                            if constexpr (PAIR) mma_f16_pair(d, x_ + k * ka, y_ + k * kbk, idesc, on);
                            else mma_f16(d, x_ + k * ka, y_ + k * kbk, idesc, on);
                            on = 1u;
                        }
                    };
                    // the small products first: less is cut off them, and off the others by theirs
                    if (b.lo) add(ad, bd + (BLOCK >> 4));
                    if (a.lo) add(ad + (BLOCK >> 4), bd);
                    add(ad, bd);
                    if constexpr (PAIR) mma_commit_pair(&sm.sums[sum % SUMS]);
                    else mma_commit(&sm.sums[sum % SUMS]);
                }
                __syncwarp();
            }
            if (!ok) break;
            if (leader) {
                if constexpr (PAIR) mma_commit_pair(&sm.empty[s]);
                else mma_commit(&sm.empty[s]);
            }
            __syncwarp();
            if (++s == STAGES) { s = 0; phase ^= 1u; }
        }
    }
    __syncwarp();
    // The sums from tensor memory into registers, a chunk at a time; zero where this share of K is empty.
    Pair sum[MINE / 2];
    const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((warp >> 2) * MINE);
    if (warp < THREADS / 32) {
#pragma unroll
        for (int k = 0; k < MINE / 2; ++k) sum[k] = pair(0.0f, 0.0f);
        const int sums = (kb1 - kb0) * (64 / SPAN);
        const int left = PAIR ? -2 : max((kb1 - kb0 - 2) * (64 / SPAN) - 1, -1);         // the sum after which the last stage is free (-1: at once)
        if (left == -1) fetch_later();
        for (int e = 0; e < sums && ok; ++e) {
            ok = __all_sync(0xffffffffu, bar_wait(&sm.sums[e % SUMS], (e / SUMS) & 1, v.wait_cycles));
            fence_after();
            if (e == left) fetch_later();
#pragma unroll
            for (int c = 0; c < MINE; c += 64) add64(mine + WIDTH * (e % SUMS) + c, sum + c / 2);
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR) arrive_even<true>(&sm.taken[e % SUMS]);
                else asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(su32(&sm.taken[e % SUMS])) : "memory");
            }
        }
    }
    ok = __syncthreads_and(ok);                                 // and the last loads have landed
    // Rows of the tile that this block finishes.  The other blocks' sums for them arrive in its shared memory, a share after the
    // other, once all are done with their rings (reading them from here instead takes 2 us more: their way is there twice).
    if constexpr (PAIR) fetch_later();
    if (split > 1 && !PAIR) cluster.sync();
    if (warp < THREADS / 32 && !idle) {
        const int r = (warp & 3) * 32 + lane, owner = r / rows;
        float *d = PAIR ? acc + ((warp >> 2) * T + r) * PITCH : acc + (rank * rows + r - owner * rows) * PITCH + (warp >> 2) * 64;
        if (shares > 1) d = cluster.map_shared_rank(d, in_cluster - rank + owner);
#pragma unroll
        for (int k = 0; k < MINE; k += 4) {
            const float2 lower = halves(sum[k / 2]), upper = halves(sum[k / 2 + 1]);
            *reinterpret_cast<float4 *>(d + k) = make_float4(lower.x, lower.y, upper.x, upper.y);
        }
    }
    if (split > 1 && !PAIR) cluster.sync();
    else __syncthreads();

    float factor = pr.factor;
    if (v.mode == GRAM && !v.later) factor *= st.gram;
    if (v.mode >= APPLY && !v.later) factor *= st.apply;
    // (tiles of Q X still read X where others are done: never into the X that this launch reads)
    uint8_t *out = v.mode == APPLY ? (v.x1 ? m.x0 : m.x1) : m.small + pr.out * slot;
#pragma unroll 1
    for (int step = 0; step < steps; ++step) {
        const int r = row_of(step), jt = tile_of(step);
        const float *mine_ = acc + ((jt - j) * T + r - r0) * PITCH + c;
        float z[8];
#pragma unroll
        for (int k = 0; k < 8; k += 4) {
            float4 y = *reinterpret_cast<const float4 *>(mine_ + k);
            for (int p = 1; p < shares; ++p) {
                const float4 o = *reinterpret_cast<const float4 *>(mine_ + k + p * rows * PITCH);
                y.x += o.x; y.y += o.y; y.z += o.z; y.w += o.w;
            }
            z[k] = y.x; z[k + 1] = y.y; z[k + 2] = y.z; z[k + 3] = y.w;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) z[k] *= factor;
        if (from[0]) {
            float f[8];
            if (step < EARLY) {
                *reinterpret_cast<float4 *>(f) = early[2 * step * THREADS];
                *reinterpret_cast<float4 *>(f + 4) = early[(2 * step + 1) * THREADS];
            } else {
                asm volatile("cp.async.wait_group %0;" ::"n"(PAIR ? ADDED - 1 : 0) : "memory");
                const uint4 *d = reinterpret_cast<const uint4 *>(added + step % ADDED * (4 * THREADS * 16));
                uint4 w[2][2] = {};
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (from[e]) {
                        w[e][0] = d[2 * e * THREADS];
                        if (from_lo) w[e][1] = d[(2 * e + 1) * THREADS];
                    }
                sum_of(w, f);
                if (PAIR) fetch(step + ADDED);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) z[k] += f[k];
        }
        if (v.mode != LEAVE) {
            if (ok) {
                uint4 h, w;
                split8(z, h, w);
                uint8_t *d = out + place(step);
                *reinterpret_cast<uint4 *>(d) = h;
                *reinterpret_cast<uint4 *>(d + lo) = w;
            }
        } else if (ok && i * T + r < m.rows) {
            const int64_t e = (int64_t)(i * T + r) * m.ldo + jt * T + c;
            const int left = m.cols - jt * T - c;
            if (v.update) {
                if (!st.finite) continue;
                float w[8];
                if (m.o_bf16) load8(static_cast<const uint16_t *>(m.out), e, left, m.ovec, w);
                else load8(static_cast<const float *>(m.out), e, left, m.ovec, w);
                const float rate = -v.lr * m.rate;
#pragma unroll
                for (int k = 0; k < 8; ++k) z[k] = clipped(w[k], rate, z[k], m.limit);
            } else if (!st.finite) {
#pragma unroll
                for (int k = 0; k < 8; ++k) z[k] = __int_as_float(0x7fc00000);
            }
            if (m.o_bf16) store8(static_cast<uint16_t *>(m.out), e, left, m.ovec, z);
            else store8(static_cast<float *>(m.out), e, left, m.ovec, z);
        }
    }
    fence_before();
    __syncwarp();
    if (PAIR) cluster.sync();                                   // no block leaves while the other's arrivals are on their way to it
    else __syncthreads();
    if (warp == ISSUER) {
        fence_after();
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;\n" ::"r"(tmem));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem));
    }
}

// ---------------------------------------------------------------------------
// Matrices whose smaller side is 64 at most: one launch
// ---------------------------------------------------------------------------
//
// A cluster takes a matrix and holds it in its blocks' shared memory, each a share of the longer side.  Its products run on
// mma.sync with fp32 values in three bf16 parts (products of parts below 2^-25 left out); every block takes the m x m
// steps by itself, the Gram matrices are added up through each other's shared memory.

constexpr int CLUSTER = 8, WARPS = THREADS / 32;
constexpr int SIDE = 64;

struct Small {
    int mt;                                  // tiles of 16 of the smaller side
    int share;                               // columns of the longer side of a block (a multiple of 64)
    int pitch, mpitch;                       // floats between rows of X and of an m x m matrix
    int mats_at, red_at;                     // floats

    __host__ __device__ static Small of(int rows, int cols) {
        const int side = rows < cols ? rows : cols, longer = rows < cols ? cols : rows;
        Small s;
        s.mt = side <= 16 ? 1 : side <= 32 ? 2 : 4;
        s.share = (longer + CLUSTER * 64 - 1) / (CLUSTER * 64) * 64;
        s.pitch = s.share + 4;               // rows begin in other banks
        s.mpitch = 16 * s.mt + 4;
        s.mats_at = 16 * s.mt * s.pitch;
        s.red_at = s.mats_at + 16 * s.mt * s.mpitch;      // the partial sums lie where all m x m matrices but the first do
        return s;
    }
    // bytes: X, five m x m matrices, or one and the warps' sums
    __host__ int64_t bytes() const {
        const int64_t m = 16 * mt, sums = (mt == 4 ? 4 : 8) * m * m, mats = 4 * m * mpitch;
        return 4 * ((int64_t)m * pitch + m * mpitch + (sums > mats ? sums : mats));
    }
};

// The parts of one fp32 row pair at k (values k, k + 1).
__device__ __forceinline__ void parts_at(const float *p, uint32_t *s) {
    const float2 v = *reinterpret_cast<const float2 *>(p);
    split2(__float_as_uint(v.x), __float_as_uint(v.y), s);
}

// Six products of parts, the smallest first.
__device__ __forceinline__ void mma_parts(float *c, const uint32_t (*a)[4], const uint32_t *b0, const uint32_t *b1) {
#pragma unroll
    for (int l = 2; l >= 0; --l)
#pragma unroll
        for (int q = 0; q <= l; ++q) mma16816(c, a[q], b0[l - q], b1[l - q]);
}

// c += them, to nearest: the tensor cores cut what they add to, so they start from zero.
__device__ __forceinline__ void add_parts(float *c, const uint32_t (*a)[4], const uint32_t *b0, const uint32_t *b1) {
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    mma_parts(sum, a, b0, b1);
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] += sum[k];
}

// out = factor P Q + b P + a I for m x m matrices in shared memory, Q symmetric.
template <int MT>
__device__ __forceinline__ void small_product(const float *P, const float *Q, float *out, int pitch, float factor, float b, float a) {
    constexpr int TILES = MT * 2 * MT, EACH = (TILES + WARPS - 1) / WARPS;          // of 16 x 8; a warp's lie in one row of tiles
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    __syncthreads();
    if (warp * EACH < TILES) {
        const int i = 16 * (warp * EACH / (2 * MT)), j0 = 8 * (warp * EACH % (2 * MT));
        float c[EACH][4];
#pragma unroll
        for (int e = 0; e < EACH; ++e)
#pragma unroll
            for (int k = 0; k < 4; ++k) c[e][k] = 0.0f;
#pragma unroll
        for (int k = 0; k < 16 * MT; k += 16) {
            uint32_t f[3][4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint32_t s[3];
                parts_at(P + (i + g + 8 * (r & 1)) * pitch + k + 2 * t + 8 * (r >> 1), s);
#pragma unroll
                for (int q = 0; q < 3; ++q) f[q][r] = s[q];
            }
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                uint32_t b0[3], b1[3];
                parts_at(Q + (j0 + 8 * e + g) * pitch + k + 2 * t, b0);
                parts_at(Q + (j0 + 8 * e + g) * pitch + k + 2 * t + 8, b1);
                add_parts(c[e], f, b0, b1);
            }
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = i + g + 8 * (k >> 1), col = j0 + 8 * e + 2 * t + (k & 1);
                out[r * pitch + col] = fmaf(factor, c[e][k], fmaf(b, P[r * pitch + col], r == col ? a : 0.0f));
            }
    }
}

// The Gram matrix of all blocks' shares of X, times `factor`, into `out` of every block.
template <int MT>
__device__ __forceinline__ void small_gram(const cg::cluster_group &cluster, const float *X, const Small &z, float *red, float *mine,
                                           float *out, float scale) {
    constexpr int M = 16 * MT, NB = MT == 4 ? 4 : 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    float c[MT][2 * MT][4];                                     // tiles of the lower triangle
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < 2 * MT; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) c[i][j][k] = 0.0f;
    for (int b = warp; b < z.share / 32; b += WARPS) {
        uint32_t p[2 * MT][3][4];
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
            const float *x = X + (8 * i + g) * z.pitch + 32 * b + 8 * t;
            const float4 u = reinterpret_cast<const float4 *>(x)[0], v = reinterpret_cast<const float4 *>(x)[1];
            const float w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
            Eight<float> e;
#pragma unroll
            for (int k = 0; k < 8; ++k) e.w[k] = __float_as_uint(w[k] * scale);
            along(e, p[i]);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                uint32_t f[3][4];
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    f[q][0] = p[2 * i][q][2 * s];
                    f[q][1] = p[2 * i + 1][q][2 * s];
                    f[q][2] = p[2 * i][q][2 * s + 1];
                    f[q][3] = p[2 * i + 1][q][2 * s + 1];
                }
#pragma unroll
                for (int j = 0; j < 2 * MT; ++j) {
                    if (j > 2 * i + 1) continue;
                    uint32_t b0[3], b1[3];
#pragma unroll
                    for (int q = 0; q < 3; ++q) { b0[q] = p[j][q][2 * s]; b1[q] = p[j][q][2 * s + 1]; }
                    add_parts(c[i][j], f, b0, b1);
                }
            }
    }
    __syncthreads();
#pragma unroll
    for (int turn = 0; turn < WARPS / NB; ++turn) {
        if (warp / NB == turn) {
            float *d = red + (warp % NB) * M * M;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 2 * MT; ++j) {
                    if (j > 2 * i + 1) continue;
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        float2 *at_ = reinterpret_cast<float2 *>(d + (16 * i + g + 4 * k) * M + 8 * j + 2 * t);
                        float2 v = make_float2(c[i][j][k], c[i][j][k + 1]);
                        if (turn > 0) { const float2 o = *at_; v.x += o.x; v.y += o.y; }
                        *at_ = v;
                    }
                }
        }
        __syncthreads();
    }
    for (int e = threadIdx.x; e < M * M; e += THREADS) {
        const int r = e / M, col = e % M;
        if (col > r) continue;
        float v[NB];
#pragma unroll
        for (int w = 0; w < NB; ++w) v[w] = red[w * M * M + e];
#pragma unroll
        for (int w = 1; w < NB; ++w) v[0] += v[w];
        mine[r * z.mpitch + col] = v[0];
    }
    cluster.sync();
    for (int e = threadIdx.x; e < M * M; e += THREADS) {
        const int r = e / M, col = e % M;
        if (col > r) continue;
        float *p = mine + r * z.mpitch + col;
        float v[CLUSTER];
#pragma unroll
        for (int k = 0; k < CLUSTER; ++k) v[k] = *cluster.map_shared_rank(p, k);
#pragma unroll
        for (int k = 1; k < CLUSTER; ++k) v[0] += v[k];
        out[r * z.mpitch + col] = v[0];
        out[col * z.mpitch + r] = v[0];
    }
    cluster.sync();                                             // `mine` may be written again
}

// X = Q X, a warp's 64 columns at a time.
template <int MT>
__device__ __forceinline__ void small_apply(float *X, const Small &z, const float *Q, float scale) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    __syncthreads();
    for (int b = warp; b < z.share / 64; b += WARPS) {
        float c[MT][8][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) c[i][j][k] = 0.0f;
#pragma unroll
        for (int k = 0; k < 16 * MT; k += 16) {
            uint32_t f[MT][3][4];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    uint32_t s[3];
                    parts_at(Q + (16 * i + g + 8 * (r & 1)) * z.mpitch + k + 2 * t + 8 * (r >> 1), s);
#pragma unroll
                    for (int q = 0; q < 3; ++q) f[i][q][r] = s[q];
                }
            const float *x = X + (k + 2 * t) * z.pitch + 64 * b + 8 * g;
#pragma unroll
            for (int j0 = 0; j0 < 8; j0 += 4) {
                float4 v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = *reinterpret_cast<const float4 *>(x + ((r & 1) + 8 * (r >> 1)) * z.pitch + j0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    auto at_ = [&](int r) { return __float_as_uint((j == 0 ? v[r].x : j == 1 ? v[r].y : j == 2 ? v[r].z : v[r].w) * scale); };
                    uint32_t b0[3], b1[3];
                    split2(at_(0), at_(1), b0);
                    split2(at_(2), at_(3), b1);
#pragma unroll
                    for (int i = 0; i < MT; ++i) add_parts(c[i][j0 + j], f[i], b0, b1);
                }
            }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float4 *d = reinterpret_cast<float4 *>(X + (16 * i + g + 8 * h) * z.pitch + 64 * b + 16 * t);
#pragma unroll
                for (int e = 0; e < 2; ++e) {                   // columns 8 e + j of the lane's 16
                    d[2 * e] = make_float4(c[i][0][2 * h + e], c[i][1][2 * h + e], c[i][2][2 * h + e], c[i][3][2 * h + e]);
                    d[2 * e + 1] = make_float4(c[i][4][2 * h + e], c[i][5][2 * h + e], c[i][6][2 * h + e], c[i][7][2 * h + e]);
                }
            }
    }
    __syncthreads();
}

template <int MT>
__device__ __forceinline__ void small_steps(const cg::cluster_group &cluster, float *smem, const Small &z, int steps, float scale) {
    constexpr int M = 16 * MT;
    float *X = smem, *mats = smem + z.mats_at, *red = smem + z.red_at;
    const int size = M * z.mpitch, stages = (steps + 2) / 3;
    float *m1 = mats + size, *m2 = m1 + size, *m3 = m2 + size, *m4 = m3 + size;
    for (int st = 0, left = steps; st < stages; ++st) {
        const int n = (left + stages - st - 1) / (stages - st);
        left -= n;
        float *A = m1, *Z = m2, *Q = m3, *W = m4;
        small_gram<MT>(cluster, X, z, red, mats, A, st == 0 ? scale : 1.0f);
        float factor = 1.0f;
        if (st == 0) {                                          // the norm from the trace
            const int lane = threadIdx.x & 31;
            float d = lane < M ? A[lane * (z.mpitch + 1)] : 0.0f;
            if (MT == 4) d += A[(lane + 32) * (z.mpitch + 1)];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
            factor = d > 0.0f ? __fdiv_rn(1.0f, __fsqrt_rn(d)) : 1.0f;
            const float inv = d > 0.0f ? __fdiv_rn(1.0f, d) : 1.0f;
            __syncthreads();
            for (int e = threadIdx.x; e < size; e += THREADS) A[e] *= inv;
        }
        for (int k = 1; k <= n; ++k) {
            float *out = k == 1 ? Q : Z;
            small_product<MT>(A, A, out, z.mpitch, CC, CB, CA);
            if (k > 1) {
                small_product<MT>(Z, Q, W, z.mpitch, 1.0f, 0.0f, 0.0f);
                float *s = Q; Q = W; W = s;
            }
            if (k < n) {
                // A <- (Z A) Z through W
                small_product<MT>(out, A, W, z.mpitch, 1.0f, 0.0f, 0.0f);
                small_product<MT>(W, out, A, z.mpitch, 1.0f, 0.0f, 0.0f);
            }
        }
        if (st == 0) {
            __syncthreads();
            for (int e = threadIdx.x; e < size; e += THREADS) Q[e] *= factor;
        }
        small_apply<MT>(X, z, Q, st == 0 ? scale : 1.0f);
    }
}

template <int N>
__global__ void __launch_bounds__(THREADS, 1) small_kernel(const __grid_constant__ Table<N> table, Step s, int steps, int update, float lr) {
    pdl_trigger();
    pdl_wait();
    extern __shared__ __align__(16) float X[];
    __shared__ uint32_t most;                                   // the largest magnitude's bits, of this block
    const Mat &m = table.m[blockIdx.x / CLUSTER];
    const int rank = blockIdx.x % CLUSTER;
    const Small z = Small::of(m.rows, m.cols);
    const int M = 16 * z.mt, l0 = rank * z.share;
    cg::cluster_group cluster = cg::this_cluster();
    if (threadIdx.x == 0) most = 0u;
    __syncthreads();
    // this block's share [M][share], from rows of the matrix or from its columns; zeros around it
    uint32_t mx = 0u;
    const int n = M * z.share;
    // place of the eight values at e0: row and column of X, of the matrix
    auto place = [&](int e0, int &i, int &l, int &r, int &c) {
        const int q = e0 / (m.tall ? M : z.share), rest = e0 - q * (m.tall ? M : z.share);
        i = m.tall ? rest : q;
        l = m.tall ? q : rest;
        r = m.tall ? l0 + l : i;
        c = m.tall ? i : l0 + l;
    };
    for (int e0 = threadIdx.x * 8; e0 < n; e0 += THREADS * 8) {
        float u[8], mom[8];
        int i, l, r, c;
        place(e0, i, l, r, c);
        value8(m, s, c < m.cols ? r : m.rows, c, u, mom);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            mx = max(mx, __float_as_uint(u[k]) & 0x7fffffffu);
            X[m.tall ? (i + k) * z.pitch + l : i * z.pitch + l + k] = u[k];
        }
    }
    mx = __reduce_max_sync(0xffffffffu, mx);
    if ((threadIdx.x & 31) == 0) atomicMax(&most, mx);
    cluster.sync();
    for (int k = 0; k < CLUSTER; ++k) mx = max(mx, *cluster.map_shared_rank(&most, k));
    const bool finite = mx < 0x7f800000u;
    // largest magnitude to [1, 2), or as near as a factor that is an fp32 number comes (the Gram matrix of 2^-22 and more is one)
    const int ex = mx == 0u ? 0 : max(ilogbf(__uint_as_float(mx)), -126);
    const float scale = ldexpf(1.0f, min(-ex, 127));
    if (finite) {
        if (z.mt == 1) small_steps<1>(cluster, X, z, steps, scale);
        else if (z.mt == 2) small_steps<2>(cluster, X, z, steps, scale);
        else small_steps<4>(cluster, X, z, steps, scale);
    }
    const float rate = -lr * m.rate;
    constexpr int LEAVES = 2;                                   // on their way at a time (one: 1.5 us more of 23)
    for (int e0 = threadIdx.x * 8; e0 < n && (finite || !update); e0 += LEAVES * THREADS * 8) {
        float w[LEAVES][8], u[LEAVES][8], mom[LEAVES][8];
        int row[LEAVES], left[LEAVES];
        int64_t at_[LEAVES];
#pragma unroll
        for (int q = 0; q < LEAVES; ++q) {
            int i, l, r, c;
            place(e0 + q * THREADS * 8, i, l, r, c);
            row[q] = r;
            left[q] = e0 + q * THREADS * 8 < n && r < m.rows ? m.cols - c : 0;
            at_[q] = r * m.ldo + c;
            if (update) {
                if (s.use) value8(m, s, left[q] > 0 ? r : m.rows, c, u[q], mom[q]);
                if (m.o_bf16) load8(static_cast<const uint16_t *>(m.out), at_[q], left[q], m.ovec, w[q]);
                else load8(static_cast<const float *>(m.out), at_[q], left[q], m.ovec, w[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < LEAVES; ++q) {
            if (left[q] <= 0) continue;
            int i, l, r, c;
            place(e0 + q * THREADS * 8, i, l, r, c);
            if (update && s.use) store8(m.mom, row[q] * m.ldm + c, left[q], m.mvec, mom[q]);
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] = finite ? X[m.tall ? (i + k) * z.pitch + l : i * z.pitch + l + k] : __int_as_float(0x7fc00000);
                if (update) v[k] = clipped(w[q][k], rate, v[k], m.limit);
            }
            if (m.o_bf16) store8(static_cast<uint16_t *>(m.out), at_[q], left[q], m.ovec, v);
            else store8(static_cast<float *>(m.out), at_[q], left[q], m.ovec, v);
        }
    }
    __syncwarp();
    cluster.sync();                                             // others read this block's magnitude
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

using namespace minw_host;

constexpr int MAX_STEPS = 10;
constexpr int SMALL_BYTES = 220 * 1024;

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Workspace bytes of one matrix: X twice, the m x m matrices.
static int64_t matrix_bytes(int rows, int cols) {
    const int64_t rb = (rows + T - 1) / T, cb = (cols + T - 1) / T, mb = rows > cols ? cb : rb;
    return (2 * rb * cb + SLOTS * mb * mb) * 4 * (int64_t)BLOCK;
}

static int64_t tiles_of(int rows, int cols) { return (int64_t)((rows + T - 1) / T) * ((cols + T - 1) / T); }

static Mat describe(const minw_matrix *g, const minw_matrix *mom, const minw_matrix *out, int k) {
    Mat m{};
    m.rows = g[k].rows;
    m.cols = g[k].cols;
    m.tall = m.rows > m.cols;
    m.g = g[k].data;
    m.ldg = g[k].ld;
    m.g_bf16 = g[k].type == MINW_BF16;
    m.gvec = reinterpret_cast<uintptr_t>(m.g) % 16 == 0 && m.ldg % (m.g_bf16 ? 8 : 4) == 0;
    if (mom) {
        m.mom = static_cast<float *>(mom[k].data);
        m.ldm = mom[k].ld;
        m.mvec = reinterpret_cast<uintptr_t>(m.mom) % 16 == 0 && m.ldm % 4 == 0;
    }
    if (out) {
        m.out = out[k].data;
        m.ldo = out[k].ld;
        m.o_bf16 = out[k].type == MINW_BF16;
        m.ovec = reinterpret_cast<uintptr_t>(m.out) % 16 == 0 && m.ldo % (m.o_bf16 ? 8 : 4) == 0;
        m.limit = out[k].limit;
        m.rate = m.tall ? sqrtf((float)m.rows / (float)m.cols) : 1.0f;
    }
    return m;
}

// Whether a matrix goes through the launch for small sides: it fits a cluster's shared memory.
static bool is_small(const minw_matrix &g) {
    return std::min(g.rows, g.cols) <= SIDE && (int64_t)g.rows * g.cols <= (1 << 24) &&
           Small::of(g.rows, g.cols).bytes() <= SMALL_BYTES;
}

// Whether those go with the large matrices of their list instead: where the launches for these have blocks to spare, that takes
// no time of its own (the ConvNet's list with its classifier and first layer 591 us, 37 more in a launch of their own), at 2e-6 to 4e-6 off
// the formula instead of 1e-6.
static bool join(const minw_matrix *g, int count) {
    const int sms = num_sms() > 0 ? num_sms() : 152;
    int64_t tiles = 0, small = 0;
    for (int k = 0; k < count; ++k) {
        if (g[k].rows == 0 || g[k].cols == 0) continue;
        const int64_t mb = (std::min(g[k].rows, g[k].cols) + T - 1) / T;
        if (is_small(g[k])) ++small;
        else tiles += mb * (mb + 1) / 2;
    }
    return tiles > 0 && (tiles + small <= sms || small <= tiles / 16);
}
static bool is_large(const minw_matrix &g, bool joined) { return g.rows > 0 && g.cols > 0 && (joined || !is_small(g)); }

// Clusters of a level on m x m matrices (gram: of the Gram products): sums along K are split into shares where that ends the
// level earlier.  A block of 64 of K takes 0.55 us, a tile's start and end 4.5, a sum over a cluster 3.5 more.  Returns the
// level's time by that.
static float shares(Mat *table, Sizes &l, Kind kind) {
    const bool gram = kind == OF_X;
    const int products = kind == TWO ? 2 : 1, sms = num_sms() > 0 ? num_sms() : 152;
    float best = 1e30f;
    for (int cluster = 1; cluster <= 8; cluster *= 2)
        // blocks of 64 of a share (where none is split: one round)
        for (int most = 1 << 20; most >= 4 && (cluster > 1 || most > 256); most = most > 256 ? 256 : most * 3 / 4) {
            int64_t clusters = 0;
            int longest = 0;
            for (int k = 0; k < l.count; ++k) {
                const int mb = table[k].mb(), kbs = gram ? 2 * std::max(table[k].rb(), table[k].cb()) : 2 * mb, tiles = mb * (mb + 1) / 2;
                int split = 1;
                while (split < cluster && (kbs + split - 1) / split > most) split *= 2;
                clusters += (tiles * split + cluster - 1) / cluster;
                longest = std::max(longest, (kbs + split - 1) / split);
            }
            // (the share of the SMs that clusters of 4 and 8 can take)
            const int64_t places = std::max(1, (int)(sms * (cluster == 8 ? 0.948f : cluster == 4 ? 0.974f : 1.0f)) / cluster), waves = (clusters * products + places - 1) / places;
            const float time = waves * (0.55f * longest + 4.5f + (cluster > 1 ? 3.5f : 0.0f));
            if (time < best * 0.999f) {
                best = time;
                int at_ = 0;
                for (int k = 0; k < l.count; ++k) {
                    const int mb = table[k].mb(), kbs = gram ? 2 * std::max(table[k].rb(), table[k].cb()) : 2 * mb, tiles = mb * (mb + 1) / 2;
                    int split = 1;
                    while (split < cluster && (kbs + split - 1) / split > most) split *= 2;
                    table[k].split[kind] = split;
                    table[k].first[kind] = at_;
                    at_ += (tiles * split + cluster - 1) / cluster;
                }
                l.clusters[kind] = at_;
                l.blocks[kind] = cluster;
            }
        }
    return best;
}

// Fills a launch's list from matrix k on; returns the next launch's first, and the workspace that it takes.  base null: that
// alone, without a plan of the levels.
static int fill(Mat *table, Sizes &l, const minw_matrix *g, const minw_matrix *mom, const minw_matrix *out, int k, int count,
                uint8_t *base, int64_t *need, bool joined) {
    l.count = l.full = l.pair_tri = l.pair_full = 0;
    l.table = reinterpret_cast<const Mat *>(base);
    int64_t used = up(CAP * sizeof(Mat), 256);
    l.stat = reinterpret_cast<Stat *>(base + used);
    used = up(used + CAP * sizeof(Stat), 256);
    int64_t tiles = 0;
    for (int e = k, n = 0; e < count && n < CAP; ++e) {         // the sums of squares lie before the matrices
        if (!is_large(g[e], joined)) continue;
        ++n;
        tiles += tiles_of(g[e].rows, g[e].cols);
    }
    l.part = reinterpret_cast<double *>(base + used);
    used = up(used + tiles * (int64_t)sizeof(double), 1024);
    for (; k < count && l.count < CAP; ++k) {
        if (!is_large(g[k], joined)) continue;
        Mat &m = table[l.count++];
        m = describe(g, mom, out, k);
        m.full0 = l.full;
        m.pair_tri0 = l.pair_tri;
        m.pair_full0 = l.pair_full;
        const int mb = m.mb();
        l.full += m.rb() * m.cb();
        l.pair_tri += (mb + 1) / 2 * ((mb + 1) / 2 + 1) / 2;
        l.pair_full += (m.rb() + 1) / 2 * ((m.cb() + 1) / 2);
        const int64_t x = (int64_t)m.rb() * m.cb() * 4 * BLOCK;
        m.x0 = base + used;
        m.x1 = m.x0 + x;
        m.small = m.x1 + x;
        used += matrix_bytes(m.rows, m.cols);
    }
    *need = used;
    if (!base) return k;
    int small_k = 0, long_k = 0;
    for (int e = 0; e < l.count; ++e) {
        small_k = std::max(small_k, 2 * table[e].mb());
        long_k = std::max(long_k, 2 * std::max(table[e].rb(), table[e].cb()));
    }
    // a pair's block of 64 of K takes 0.85 us, its tiles' start and end 7; those of a tile where there are several a block, 0.62 and 5
    const int sms = num_sms() > 0 ? num_sms() : 152;
    auto pairs = [&](int64_t clusters, int k) { return (2 * clusters + sms - 1) / sms * (0.85f * k + 7.0f); };
    // (five steps: 2 Gram levels, 12 of one product, one of two)
    const float of_x = shares(table, l, OF_X), one = shares(table, l, ONE), two = shares(table, l, TWO);
    l.pairs = 2 * pairs(l.pair_tri, long_k) + 12 * pairs(l.pair_tri, small_k) + pairs(2 * (int64_t)l.pair_tri, small_k) < 2 * of_x + 12 * one + two;
    l.pairs_x = pairs(l.pair_full, small_k) < (l.full + sms - 1) / sms * (0.62f * small_k + 5.0f);
    return k;
}

static minw_status check(const minw_matrix *g, const minw_matrix *o, int count, bool floats) {
    for (int k = 0; k < count; ++k) {
        const minw_matrix &m = o ? o[k] : g[k];
        if (m.type != MINW_F32 && (m.type != MINW_BF16 || floats)) return MINW_EINVAL;
        if (m.rows < 0 || m.cols < 0 || m.rows != g[k].rows || m.cols != g[k].cols || m.ld < m.cols) return MINW_EINVAL;
        if (m.rows > 0 && m.cols > 0 && !m.data) return MINW_EINVAL;
        if (reinterpret_cast<uintptr_t>(m.data) % (m.type == MINW_BF16 ? 2 : 4) != 0) return MINW_EINVAL;
    }
    return MINW_OK;
}

// Tiles of a launch stay within 32 bits, a side within what an index of a tile's row of blocks takes.
static bool sizes_fit(const minw_matrix *g, int count) {
    int64_t tiles = 0;
    for (int k = 0; k < count; ++k) {
        if (g[k].rows > (1 << 22) || g[k].cols > (1 << 22) || std::min(g[k].rows, g[k].cols) > (1 << 15)) return false;
        tiles += tiles_of(g[k].rows, g[k].cols);
    }
    return tiles < (1 << 26);
}

template <int N>
static cudaError_t launch(const Sizes &l, Level v, const Table<N> &own, cudaStream_t s) {
    const Kind kind = v.mode == GRAM ? OF_X : v.products == 1 ? ONE : TWO;
    const bool tri = v.mode <= MUL;
    const int64_t pairs = tri ? (int64_t)l.pair_tri * v.products : l.pair_full;
    const bool pair = tri ? l.pairs : l.pairs_x;
    v.upper = l.pairs;
    v.split = pair ? 2 : tri ? l.blocks[kind] : 1;
    const int64_t clusters = pair ? pairs : tri ? (int64_t)l.clusters[kind] * v.products : l.full;
    v.wait_cycles = (long long)plan_options().wait_cycles;
    auto kern = pair ? product_kernel<true, N> : product_kernel<false, N>;
    const int smem = STAGES * (int)STAGE + EARLY * 2 * THREADS * 16 + 1024;                               // (as much for pairs)
    if (!allow_shared(reinterpret_cast<const void *>(kern), smem)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(clusters * v.split));
    cfg.blockDim = dim3(THREADS + 64);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)v.split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    max_shared_carveout(reinterpret_cast<const void *>(kern));
    return cudaLaunchKernelEx(&cfg, kern, l, v, own);
}

// All steps of one list; own: its descriptions for the launches of products (none: read from the workspace).
template <int M, int N>
static minw_status chain(const Table<M> &table, const Table<N> &own, const Sizes &l, const Step &step, int steps, bool x_lo, bool update,
                         float lr, cudaStream_t s) {
    const dim3 tiles((unsigned)l.full);
    if (launch_pdl_stream(false, squares_kernel<M>, tiles, dim3(THREADS), 0, s, table, l, step) != cudaSuccess) return launch_failed();
    if (launch_pdl_stream(false, enter_kernel, tiles, dim3(THREADS), 0, s, l, step, x_lo ? 1 : 0) !=
        cudaSuccess)
        return launch_failed();
    // powers of two at which the m x m matrices are held: A, Z A below 1.447, W below 2.81, R after k steps below 3.4446^k
    const int SA = 15, SW = 14;
    static const int SR[4] = {0, 14, 12, 10};
    auto two = [](int e) { return ldexpf(1.0f, e); };
    const int stages = (steps + 2) / 3;
    for (int st = 0, left = steps; st < stages; ++st) {
        const int n = (left + stages - st - 1) / (stages - st);                       // 3 + 2 of five
        left -= n;
        const bool last = st + 1 == stages;
        int A = 0, R = -1;
        float q = CA;                                                                 // Q = q I + R
        Level v{};
        v.later = st > 0;
        v.x1 = st & 1;
        v.x_lo = st > 0 || x_lo;
        v.mode = GRAM;
        v.products = 1;
        v.pr[0] = {0, 0, A, two(SA - 30), {-1, -1}, {}};
        if (launch(l, v, own, s) != cudaSuccess) return launch_failed();
        for (int k = 1; k <= n; ++k) {
            const int W = k == 1 ? 4 : 2;                                             // the first W is R
            Level p{};
            p.mode = MUL;
            p.products = 1;
            p.pr[0] = {A, A, W, CC * two(SW - 2 * SA), {A, -1}, {CB * two(SW - SA), 0.0f}};
            if (launch(l, p, own, s) != cudaSuccess) return launch_failed();
            Level w{};
            w.mode = MUL;
            if (k < n) w.pr[w.products++] = {W, A, 3, two(-SW), {A, -1}, {CA, 0.0f}};                     // Z A = W A + a A
            if (k > 1) {                                                              // Z Q = W R + a R + q W, and a q I
                w.pr[w.products++] = {W, R, R ^ 1, two(SR[k] - SW - SR[k - 1]), {R, W}, {CA * two(SR[k] - SR[k - 1]), q * two(SR[k] - SW)}};
                q *= CA;
            }
            R = k == 1 ? 4 : R ^ 1;
            if (w.products > 0 && launch(l, w, own, s) != cudaSuccess) return launch_failed();
            if (k < n) {
                w.products = 1;
                w.pr[0] = {3, W, A ^ 1, two(-SW), {3, -1}, {CA, 0.0f}};               // (Z A) Z
                if (launch(l, w, own, s) != cudaSuccess) return launch_failed();
                A ^= 1;
            }
        }
        Level e{};
        e.mode = last ? LEAVE : APPLY;
        e.products = 1;
        e.later = st > 0;
        e.x1 = st & 1;
        e.x_lo = st > 0 || x_lo;
        e.update = update;
        e.lr = lr;
        e.pr[0] = {R, R, 0, two((last ? 0 : 15) - SR[n] - 15), {-1, -1}, {q * two(last ? -15 : 0), 0.0f}};
        if (launch(l, e, own, s) != cudaSuccess) return launch_failed();
    }
    return launch_status();
}

template <int N>
static cudaError_t launch_small(const Table<N> &table, int count, int bytes, const Step &step, int steps, bool update, float lr,
                                cudaStream_t s) {
    auto kern = small_kernel<N>;
    if (!allow_shared(reinterpret_cast<const void *>(kern), SMALL_BYTES)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(count * CLUSTER));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = (size_t)bytes;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CLUSTER;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, table, step, steps, update ? 1 : 0, lr);
}

static minw_status run(const minw_matrix *g, const minw_matrix *mom, const minw_matrix *out, int count, int steps,
                       const Step &step, bool update, float lr, uint8_t *ws, cudaStream_t s) {
    bool x_lo = step.use != 0;                                  // bf16 gradients are fp16 numbers but for the smallest
    for (int k = 0; k < count; ++k) x_lo = x_lo || g[k].type == MINW_F32;
    const bool joined = join(g, count);
    Table<CAP> table;
    for (int k = 0; k < count;) {
        int n = 0;
        int64_t bytes = 0;
        for (; k < count && n < CAP; ++k) {
            if (g[k].rows == 0 || g[k].cols == 0 || is_large(g[k], joined)) continue;
            table.m[n++] = describe(g, mom, out, k);
            bytes = std::max(bytes, Small::of(g[k].rows, g[k].cols).bytes());
        }
        if (n == 0) break;
        cudaError_t e;
        if (n <= FEW) {
            Table<FEW> few;
            std::copy(table.m, table.m + n, few.m);
            e = launch_small(few, n, (int)bytes, step, steps, update, lr, s);
        } else {
            e = launch_small(table, n, (int)bytes, step, steps, update, lr, s);
        }
        if (e != cudaSuccess) return launch_failed();
    }
    Sizes l;
    for (int k = 0; k < count;) {
        int64_t need;
        k = fill(table.m, l, g, mom, out, k, count, ws, &need, joined);
        if (l.count == 0) break;
        minw_status st;
        if (l.count <= FEW) {
            Table<FEW> few;
            std::copy(table.m, table.m + l.count, few.m);
            st = chain(few, few, l, step, steps, x_lo, update, lr, s);
        } else {
            st = chain(table, Table<0>{}, l, step, steps, x_lo, update, lr, s);
        }
        if (st != MINW_OK) return st;
    }
    return launch_status();
}

}  // namespace orth

int take_orth_error() {
    int flag = 0;
    if (cudaMemcpyFromSymbol(&flag, g_orth_error, sizeof(int)) != cudaSuccess) return -1;
    if (flag) {
        const int zero = 0;
        if (cudaMemcpyToSymbol(g_orth_error, &zero, sizeof(int)) != cudaSuccess) return -1;
    }
    return flag ? 1 : 0;
}

}  // namespace minw

using namespace minw;
using namespace minw_host;

extern "C" {

size_t minw_orthogonal_workspace_bytes(const minw_matrix *grads, int32_t count) {
    if (count < 0 || (count > 0 && !grads) || orth::check(grads, nullptr, count, false) != MINW_OK ||
        !orth::sizes_fit(grads, count))
        return 0;
    orth::Table<orth::CAP> table;
    orth::Sizes l;
    const bool joined = orth::join(grads, count);
    int64_t most = 16;
    for (int k = 0; k < count;) {
        int64_t need;
        k = orth::fill(table.m, l, grads, nullptr, nullptr, k, count, nullptr, &need, joined);
        most = std::max(most, need);
    }
    return (size_t)most;
}

static minw_status orthogonal(const minw_matrix *grads, const minw_matrix *mom, const minw_matrix *out, int32_t count,
                              int32_t steps, const orth::Step &step, bool update, float lr, void *ws, size_t bytes,
                              void *stream) {
    if (count < 0 || (count > 0 && (!grads || !out)) || steps < 1 || steps > orth::MAX_STEPS) return MINW_EINVAL;
    if (orth::check(grads, nullptr, count, false) != MINW_OK || orth::check(grads, out, count, false) != MINW_OK ||
        (mom && orth::check(grads, mom, count, true) != MINW_OK))
        return MINW_EINVAL;
    for (int k = 0; k < count; ++k) {
        if (update && !(out[k].limit >= 0.0f)) return MINW_EINVAL;
        if (grads[k].rows == 0 || grads[k].cols == 0) continue;
        // only an orthogonalised matrix may be its gradient
        const bool same = out[k].data == grads[k].data;
        if (same && (update || out[k].type != grads[k].type || out[k].ld != grads[k].ld)) return MINW_EINVAL;
        if (mom && (mom[k].data == grads[k].data || mom[k].data == out[k].data)) return MINW_EINVAL;
    }
    if (!orth::sizes_fit(grads, count)) return MINW_EUNSUPPORTED;
    bool some = false;
    for (int k = 0; k < count; ++k) some = some || (grads[k].rows > 0 && grads[k].cols > 0);
    if (!some) return MINW_OK;
    if (!ws || !aligned16(ws) || bytes < minw_orthogonal_workspace_bytes(grads, count)) return MINW_EINVAL;
    return orth::run(grads, mom, out, count, steps, step, update, lr, static_cast<uint8_t *>(ws), (cudaStream_t)stream);
}

minw_status minw_orthogonalize(const minw_matrix *grads, const minw_matrix *out, int32_t count, int32_t steps,
                               void *workspace, size_t workspace_bytes, void *stream) {
    return orthogonal(grads, nullptr, out, count, steps, orth::Step{0.0f, 0, 0}, false, 0.0f, workspace, workspace_bytes,
                      stream);
}

minw_status minw_sgd_orthogonal(const minw_matrix *weights, const minw_matrix *momenta, const minw_matrix *grads,
                                int32_t count, int32_t steps, float momentum, int32_t nesterov, float lr, void *workspace,
                                size_t workspace_bytes, void *stream) {
    if (!isfinite(lr) || !isfinite(momentum) || (count > 0 && !weights)) return MINW_EINVAL;
    return orthogonal(grads, momenta, weights, count, steps, orth::Step{momentum, momenta ? 1 : 0, nesterov ? 1 : 0}, true,
                      lr, workspace, workspace_bytes, stream);
}

}  // extern "C"
