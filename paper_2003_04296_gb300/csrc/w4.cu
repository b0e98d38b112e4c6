// w4.cu -- 4-bit weights with group scales: packing, and products of a few
// vectors with them.
//
// A product of T vectors with O x K weights reads O K / 2 bytes of codes and
// O K 2 / group of scales, and little else: for a few vectors it is bound by
// memory, at about 2.7 instructions per weight and lane of the whole chip.  So
// the codes are turned into bf16 two at a time -- code | 0x4300 is 128 + code
// in bf16, minus 136 is the level, both exact -- and the multiply-adds run on
// mma.sync (bf16 x bf16, fp32 sums): the weights are its 16-row operand, the
// vectors its 8 columns.  A tile of the tcgen05 tensor cores has 128 rows and
// takes both operands from shared memory, which the unpacked weights would
// have to be written to first, at four times their packed bytes.  Measured, one
// vector: 16384 x 16384 in 32.7 us, 4.2 TB/s, 1024 x 8192 in 4.2 us (latency);
// eight: 8192 x 8192 in 12.6.  No unit is full in the first (counters, shares of
// the whole launch): instructions issue in 48 % of the clocks, the integer pipe
// is busy 43 %, the shared memory's reads 54 %, DRAM 50 %.  14 warps an SM, three
// to a scheduler, hide too little of each other's waits: for the integer pipe's
// turn 17 % of a warp's time, for fixed latencies 13 %, at the barriers around
// the vectors' staging 11 %, for data 6 %.
//
// A lane reads 16 bytes of codes of two rows: 32 values each, four groups of
// eight.  The layout puts the eight values 32 j + 8 t of a block of 128 into
// word j of lane t's 16 bytes, so that word j of the four lanes of a row is a
// group of 32 consecutive values (the finest scales), and the pairs (2p, 2p + 1)
// of a word's values into nibbles p and p + 4, so that a shift and a mask give
// a register of two consecutive values, against which a row of x stands as it
// lies in memory.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "kernels.cuh"
#include "values.cuh"
#include "w4.cuh"

namespace cg = cooperative_groups;

namespace minw {
namespace w4 {

constexpr int THREADS = 256;          // of a packing block

// ---------------------------------------------------------------------------
// Packing
// ---------------------------------------------------------------------------

// S lanes per row and group: the group's largest magnitude, its scale, its codes.  Single loads, w read twice: once per
// set of weights (16384 x 16384 fp32 469 us).
template <typename T, int S>
__global__ void __launch_bounds__(THREADS) pack_kernel(const T *__restrict__ w, int O, int K, int Kp, int group,
                                                       int quantize, QParams q, const float *channel_scale,
                                                       uint8_t *__restrict__ codes, uint16_t *__restrict__ scales) {
    pdl_wait();          // lets no dependent start early: its output is weights
    const int covered = (Kp + group - 1) / group, groups = (K + group - 1) / group;
    const int64_t at = ((int64_t)blockIdx.x * THREADS + threadIdx.x) / S;
    const int sl = (int)threadIdx.x % S;
    const bool live = at < (int64_t)O * covered;
    const int o = live ? (int)(at / covered) : 0, g = live ? (int)(at % covered) : 0;
    const int k0 = g * group, k1 = min(K, k0 + group), kp1 = min(Kp, k0 + group);
    const T *row = w + (int64_t)o * K;
    auto value = [&](int k) {
        Vec<T, 1> v;
        v.load(row + k);
        return v.get(0);
    };
    float scale = 1.0f;
    if (!quantize) {
        uint32_t m = 0;                     // magnitudes as integers: monotone, a NaN above all
        if (live)
            for (int k = k0 + 8 * sl; k < k1; k += 8 * S)
                for (int i = 0; i < 8 && k + i < k1; ++i) m = max(m, __float_as_uint(value(k + i)) & 0x7fffffffu);
#pragma unroll
        for (int d = S / 2; d > 0; d >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
        scale = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(__uint_as_float(m), 7.0f)));
    }
    if (!live) return;
    if (sl == 0 && g < groups) scales[(int64_t)o * groups + g] = __bfloat16_as_ushort(__float2bfloat16_rn(scale));
    const bool some = scale > 0.0f && scale <= 3.4e38f;
    const float cs = quantize ? (channel_scale ? channel_scale[o] : q.scale) : 1.0f;
    uint32_t *out = reinterpret_cast<uint32_t *>(codes + (int64_t)o * (Kp / 2));
    for (int k = k0 + 8 * sl; k < kp1; k += 8 * S) {
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int code = 8;
            if (k + i < k1) {
                const float v = value(k + i);
                if (quantize) code = 8 + level_units(v * cs, q);
                else if (some) code = 8 + (int)fminf(7.0f, fmaxf(-7.0f, rintf(__fdiv_rn(v, scale))));
            }
            word |= (uint32_t)code << (4 * (i / 2 + 4 * (i % 2)));
        }
        const int e = (k & 127) >> 3;                                  // 8 values 32 j + 8 t: e = 4 j + t
        out[(k >> 7) * 16 + 4 * (e & 3) + (e >> 2)] = word;
    }
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------

struct Args {
    const void *x;
    int64_t ldx, ldy;
    const uint8_t *codes;
    const uint16_t *scales;
    const float *scale, *shift;
    const float *add;                  // [T][O], or null
    void *y;
    int T, O, K, nb, groups, group;    // nb: blocks of 128 values of a row
    int x_bf16, y_bf16, act;
    int parts, tokens;                 // columns of a vector (1, or 3 for fp32), vectors of a pass
    int wr, wk;                        // warps side by side along the rows, and along K
    int split, upc;                    // CTAs of a cluster (they split K), units of two blocks of each
    int xunits;                        // units whose x and scales are in shared memory at a time
    int xpitch, scale_pitch;           // values between columns of x, and between rows of scales, there
    int scale_at, ring_at;             // where scales and codes lie (bytes)
    Div by_row, by_eights;             // loads of 16 bytes of a column's x, of a row's scales
    Div by_blocks;                     // blocks of 128 values per group (groups of 128 and more)
};

__device__ __forceinline__ uint32_t levels(uint32_t word, int p) {
    uint32_t v = word >> (4 * p);
    asm("lop3.b32 %0, %0, %1, %2, 0xea;" : "+r"(v) : "r"(0x000f000fu), "r"(0x43004300u));     // (v & ..) | ..: 128 + code
    asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(v) : "r"(0xc308c308u));                            // - 136
    return v;
}

__device__ __forceinline__ void mma(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Three bf16 values whose sum is v: its leading 8 bits, the next 8, the rest.  Infinities and NaN stay in the first.
__device__ __forceinline__ void split3(float v, uint16_t *p) {
    const uint32_t b = __float_as_uint(v);
    if ((b & 0x7f800000u) == 0x7f800000u) {
        p[0] = (uint16_t)((b >> 16) | ((b & 0x007fffffu) ? 0x40u : 0u));
        p[1] = p[2] = 0;
        return;
    }
    const float r = v - __uint_as_float(b & 0xffff0000u);
    const uint32_t m = __float_as_uint(r);
    p[0] = (uint16_t)(b >> 16);
    p[1] = (uint16_t)(m >> 16);
    p[2] = __bfloat16_as_ushort(__float2bfloat16_rn(r - __uint_as_float(m & 0xffff0000u)));
}

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy16(uint16_t *dst, const void *src, int bytes) {
    copy16((uint32_t)__cvta_generic_to_shared(dst), src, bytes);
}

// A value that is read before the wait (a.add), else after it.
template <typename V>
__device__ __forceinline__ V early(const Args &a, const V *p) { return a.add ? __ldcg(p) : *p; }

// The pass's vectors from value k0 on into shared memory, xunits units of them: columns of xpitch values (the 64
// bytes over put the eight columns of a tile into different banks), zero past K.
__device__ __forceinline__ void stage_x(const Args &a, uint16_t *xs, int t0, int tokens, int k0) {
    const int threads = blockDim.x, per_row = a.by_row.d, all = tokens * per_row;
    if (a.x_bf16) {
        const uint16_t *x = static_cast<const uint16_t *>(a.x) + (int64_t)t0 * a.ldx + k0;
        const bool wide = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && a.ldx % 8 == 0;
        for (int e = threadIdx.x; e < all; e += threads) {           // eights
            const int t = a.by_row.div(e), k = 8 * (e - t * per_row), left = a.K - k0 - k;
            const uint16_t *src = x + t * a.ldx + k;
            uint16_t *dst = xs + t * a.xpitch + k;
            if (wide) {
                copy16(dst, left > 0 ? src : x, left >= 8 ? 16 : left > 0 ? 2 * left : 0);
            } else {
                uint16_t v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = i < left ? early(a, src + i) : (uint16_t)0;
                *reinterpret_cast<uint4 *>(dst) = make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16,
                                                             v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16);
            }
        }
    } else {
        constexpr int U = 4;                                         // loads in flight
        const float *x = static_cast<const float *>(a.x) + (int64_t)t0 * a.ldx + k0;
        const bool wide = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && a.ldx % 4 == 0;
        for (int e0 = threadIdx.x; e0 < all; e0 += U * threads) {    // fours
            float4 v[U];
            int at[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = e0 + u * threads, t = a.by_row.div(e), k = 4 * (e - t * per_row), left = a.K - k0 - k;
                v[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                at[u] = 3 * t * a.xpitch + k;
                if (e >= all) continue;
                const float *src = x + t * a.ldx + k;
                if (wide && left >= 4) {
                    v[u] = early(a, reinterpret_cast<const float4 *>(src));
                } else {
                    if (left > 0) v[u].x = early(a, src + 0);
                    if (left > 1) v[u].y = early(a, src + 1);
                    if (left > 2) v[u].z = early(a, src + 2);
                    if (left > 3) v[u].w = early(a, src + 3);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (e0 + u * threads >= all) break;
                uint16_t p[4][3];
                split3(v[u].x, p[0]);
                split3(v[u].y, p[1]);
                split3(v[u].z, p[2]);
                split3(v[u].w, p[3]);
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    *reinterpret_cast<uint2 *>(xs + at[u] + i * a.xpitch) =
                        make_uint2(p[0][i] | (uint32_t)p[1][i] << 16, p[2][i] | (uint32_t)p[3][i] << 16);
            }
        }
    }
}

// The scales of the CTA's rows from group g0 on, scale_pitch of each; zero for groups past the last (they hold padding
// only).
__device__ __forceinline__ void stage_scales(const Args &a, uint16_t *ss, int row0, int g0) {
    const int threads = blockDim.x, eights = a.by_eights.d, all = a.wr * 16 * eights;
    const bool wide = (reinterpret_cast<uintptr_t>(a.scales + g0) & 15) == 0 && a.groups % 8 == 0;
    for (int e = threadIdx.x; e < all; e += threads) {
        const int r = a.by_eights.div(e), k = 8 * (e - r * eights), left = a.groups - g0 - k;
        const uint16_t *src = a.scales + (int64_t)min(row0 + r, a.O - 1) * a.groups + g0 + k;
        uint16_t *dst = ss + 8 * e;
        if (wide) {
            copy16(dst, left > 0 ? src : a.scales + g0, left >= 8 ? 16 : left > 0 ? 2 * left : 0);
        } else {
            uint16_t v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < left ? early(a, src + i) : (uint16_t)0;
            *reinterpret_cast<uint4 *>(dst) = make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16,
                                                         v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16);
        }
    }
}

constexpr int WARPS = 8;              // of a CTA, at most
// Units of a warp's ring in shared memory, one of them in use, the others on their way (asynchronous copies): for one
// tile of columns, and for several, which leave more time for each.
__host__ __device__ constexpr int ring_of(int NT) { return NT == 1 ? 4 : 2; }
constexpr int UNIT_BYTES = 2048;      // 16 rows x two blocks (128 bytes of a row side by side)

// NT: tiles of 8 columns; FL: words of a lane's four that share a scale (1, 2, 4 for groups of 32, 64, 128 and more).
template <int NT, int FL>
__global__ void __launch_bounds__(32 * WARPS, 2) matvec_kernel(Args a) {
    pdl_trigger();
    // What the kernel before this one wrote (add) is needed at the end alone.  Until then x, codes and scales are read through
    // L2, where they lay before that kernel let this one start: what an SM's own cache holds is certain to be new only after a wait.
    if (!a.add) pdl_wait();
    constexpr int RING = ring_of(NT);
    extern __shared__ __align__(16) uint8_t smem[];
    uint16_t *xs = reinterpret_cast<uint16_t *>(smem), *ss = reinterpret_cast<uint16_t *>(smem + a.scale_at);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int wr = warp % a.wr, wk = warp / a.wr;
    const int rank = blockIdx.x % a.split, tile = blockIdx.x / a.split;
    const int t0 = blockIdx.y * a.tokens, tokens = min(a.tokens, a.T - t0), cols = tokens * a.parts;
    const int row0 = tile * a.wr * 16, row = row0 + wr * 16 + g;
    const int64_t pitch = (int64_t)a.nb * 64;
    // rows past the last repeat it and are not stored
    const uint8_t *w0 = a.codes + min(row, a.O - 1) * pitch + 16 * t, *w1 = a.codes + min(row + 8, a.O - 1) * pitch + 16 * t;
    const int first = rank * a.upc, last = min((a.nb + 1) / 2, first + a.upc);
    uint8_t *ring = smem + a.ring_at + warp * (RING * UNIT_BYTES) + lane * 16;
    const uint32_t ring_copy = (uint32_t)__cvta_generic_to_shared(ring);
    const int step = a.wk * 128;
    int next = first + wk, fetched = 0, used = 0;                        // slots as offsets in bytes
    w0 += next * 128;
    w1 += next * 128;
    auto fetch = [&]() {                                                 // a lane reads back what it has copied itself
        if (next < last) {
            // a block past the last: zeros (against zeros of x)
            const int bytes = 2 * next + 1 < a.nb ? 16 : 0, more = bytes * 4;
            const uint32_t d = ring_copy + fetched;
            copy16(d, w0, 16);
            copy16(d + 512, w1, 16);
            copy16(d + 1024, w0 + more, bytes);
            copy16(d + 1536, w1 + more, bytes);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        next += a.wk;
        w0 += step;
        w1 += step;
        fetched = (fetched + UNIT_BYTES) & (RING * UNIT_BYTES - 1);
    };

    float tot[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) tot[n][i] = 0.0f;
#pragma unroll
    for (int d = 0; d < RING - 1; ++d) fetch();

    for (int c0 = first; c0 < last; c0 += a.xunits) {
        const int b0 = 2 * c0, xpitch = a.xpitch;
        const int g0 = FL == 4 ? a.by_blocks.div(b0) : b0 * (4 / FL);
        __syncthreads();
        stage_x(a, xs, t0, tokens, b0 * 128);
        stage_scales(a, ss, row0, g0);
        if (threadIdx.x < 32) *reinterpret_cast<uint4 *>(xs + cols * xpitch + 8 * threadIdx.x) = make_uint4(0, 0, 0, 0);
        asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        // this lane's column of each tile, at its values of the unit; a column past the last is 256 zeros
        const uint16_t *xr[NT];
        int xstep[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const bool live = n * 8 + g < cols;
            xr[n] = xs + (live ? (n * 8 + g) * xpitch + wk * 256 : cols * xpitch) + 8 * t;
            xstep[n] = live ? a.wk * 256 : 0;
        }
        const uint16_t *sr = ss + (wr * 16 + g) * a.scale_pitch - g0;
        const int end = min(c0 + a.xunits, last);
        for (int u = c0 + wk; u < end; u += a.wk) {
            asm volatile("cp.async.wait_group %0;" ::"n"(RING - 2) : "memory");
            fetch();
            const uint8_t *d = ring + used;
            used = (used + UNIT_BYTES) & (RING * UNIT_BYTES - 1);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint4 u0 = *reinterpret_cast<const uint4 *>(d + b * 1024);
                const uint4 u1 = *reinterpret_cast<const uint4 *>(d + b * 1024 + 512);
                const uint32_t q0[4] = {u0.x, u0.y, u0.z, u0.w}, q1[4] = {u1.x, u1.y, u1.z, u1.w};
                const uint16_t *sb = sr + (FL == 4 ? a.by_blocks.div(2 * u + b) : (2 * u + b) * (4 / FL));
                // a scale's words in one sum, the four words of a long group in two (shorter chains of dependent products)
                constexpr int SUMS = FL == 4 ? 2 : 1;
                float acc[SUMS][NT][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j % FL == 0) {
#pragma unroll
                        for (int h = 0; h < SUMS; ++h)
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int i = 0; i < 4; ++i) acc[h][n][i] = 0.0f;
                    }
                    const int h = j % SUMS;
                    uint32_t a0[4], a1[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        a0[p] = levels(q0[j], p);
                        a1[p] = levels(q1[j], p);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(xr[n] + 128 * b + 32 * j);
                        mma(acc[h][n], a0[0], a1[0], a0[1], a1[1], v.x, v.y);
                        mma(acc[h][n], a0[2], a1[2], a0[3], a1[3], v.z, v.w);
                    }
                    if (j % FL == FL - 1) {
                        const float f0 = __uint_as_float((uint32_t)sb[j / FL] << 16);
                        const float f1 = __uint_as_float((uint32_t)sb[8 * a.scale_pitch + j / FL] << 16);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float sum = SUMS == 1 ? acc[0][n][i] : acc[0][n][i] + acc[SUMS - 1][n][i];
                                tot[n][i] = fmaf(i < 2 ? f0 : f1, sum, tot[n][i]);
                            }
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) xr[n] += xstep[n];
        }
    }

    // the warps' sums [warp][16 rows][8 NT columns], added up over the warps along K into the first wr, then over the
    // cluster; all in a fixed order
    constexpr int CW = 8 * NT;
    float *red = reinterpret_cast<float *>(smem);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float *d = red + (warp * 16 + g) * CW + n * 8 + 2 * t;
        *reinterpret_cast<float2 *>(d) = make_float2(tot[n][0], tot[n][1]);
        *reinterpret_cast<float2 *>(d + 8 * CW) = make_float2(tot[n][2], tot[n][3]);
    }
    __syncthreads();
    const int rows = a.wr * 16, size = rows * CW;
    if (a.wk > 1) {
        for (int e = threadIdx.x; e < size; e += blockDim.x) {
            float v[WARPS];
#pragma unroll
            for (int k = 0; k < WARPS; ++k) v[k] = k < a.wk ? red[k * size + e] : 0.0f;
#pragma unroll
            for (int k = 1; k < WARPS; ++k) v[0] += v[k];
            red[e] = v[0];
        }
    }
    cg::cluster_group cluster = cg::this_cluster();
    if (a.split > 1) cluster.sync();
    else __syncthreads();
    if (a.add) pdl_wait();
    const int each = (rows + a.split - 1) / a.split, rr0 = rank * each, rr1 = min(rows, rr0 + each);
    for (int e = threadIdx.x; e < (rr1 - rr0) * tokens; e += blockDim.x) {
        const int q = e / tokens, tk = e - q * tokens, r = rr0 + q, o = row0 + r;
        if (o >= a.O) continue;
        float sum = 0.0f;
        for (int i = a.parts - 1; i >= 0; --i) {                      // the smallest part first
            float *at = red + r * CW + tk * a.parts + i;
            float v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c)
                v[c] = a.split == 1 ? (c == 0 ? *at : 0.0f) : c < a.split ? *cluster.map_shared_rank(at, c) : 0.0f;
#pragma unroll
            for (int c = 1; c < 8; ++c) v[0] += v[c];
            sum += v[0];
        }
        if (a.add) sum += a.add[(int64_t)(t0 + tk) * a.O + o];
        float z = fmaf(sum, a.scale ? a.scale[o] : 1.0f, a.shift ? a.shift[o] : 0.0f);
        with_act(a.act, [&](auto act) { z = act_value<act.value>(z); });
        const int64_t at = (int64_t)(t0 + tk) * a.ldy + o;
        if (a.y_bf16) static_cast<uint16_t *>(a.y)[at] = __bfloat16_as_ushort(__float2bfloat16_rn(z));
        else static_cast<float *>(a.y)[at] = z;
    }
    if (a.split > 1) {
        cluster_done_reading();
        cluster_leave();
    }
}

using namespace minw_host;

static bool valid_group(int g) { return g == 32 || g == 64 || (g > 0 && g % 128 == 0); }

template <typename T>
static cudaError_t pack(const void *w, int O, int K, int Kp, int group, const minw_quant *q, const float *cs,
                        uint8_t *codes, uint16_t *scales, cudaStream_t s) {
    const int S = group >= 256 ? 32 : group / 8;
    const int64_t threads = (int64_t)O * ((Kp + group - 1) / group) * S;
    const QParams p = q ? to_qparams(q) : QParams{};
    auto kern = S == 32 ? pack_kernel<T, 32> : S == 16 ? pack_kernel<T, 16> : S == 8 ? pack_kernel<T, 8>
                                                                                     : pack_kernel<T, 4>;
    return launch_pdl_stream(false, kern, dim3((unsigned)((threads + THREADS - 1) / THREADS)), dim3(THREADS), 0, s,
                             static_cast<const T *>(w), O, K, Kp, group, q ? 1 : 0, p, cs, codes, scales);
}

template <int NT, int FL>
static cudaError_t launch(const Args &a, dim3 grid, size_t smem, cudaStream_t s) {
    auto kern = matvec_kernel<NT, FL>;
    if (!allow_shared(reinterpret_cast<const void *>(kern), 112 * 1024)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(32u * a.wr * a.wk);
    cfg.dynamicSmemBytes = smem;
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

template <int NT>
static cudaError_t launch_group(const Args &a, int group, dim3 grid, size_t smem, cudaStream_t s) {
    return group == 32 ? launch<NT, 1>(a, grid, smem, s) : group == 64 ? launch<NT, 2>(a, grid, smem, s)
                                                                       : launch<NT, 4>(a, grid, smem, s);
}

minw_status check(const void *x, int x_type, int64_t ldx, int64_t T, const uint8_t *codes, const uint16_t *scales, int O, int K,
                  int group, const float *scale, const float *shift, int act, const void *y, int y_type, int64_t ldy) {
    if (!codes || !scales || (T != 0 && (!x || !y)) || T < 0 || O < 1 || K < 1 || ldx < K || ldy < O) return MINW_EINVAL;
    if (!valid_group(group) || act < MINW_ACT_NONE || act > MINW_ACT_SILU) return MINW_EINVAL;
    if ((x_type != MINW_F32 && x_type != MINW_BF16) || (y_type != MINW_F32 && y_type != MINW_BF16)) return MINW_EINVAL;
    if (!aligned16(codes) || reinterpret_cast<uintptr_t>(scales) % 2 != 0 || !on_floats(scale, shift) ||
        reinterpret_cast<uintptr_t>(x) % (x_type == MINW_BF16 ? 2 : 4) != 0 ||
        reinterpret_cast<uintptr_t>(y) % (y_type == MINW_BF16 ? 2 : 4) != 0)
        return MINW_EINVAL;
    if (K > (1 << 28) || group > (1 << 28) || O > (1 << 28)) return MINW_EUNSUPPORTED;
    return MINW_OK;
}

minw_status matvec(const void *x, int x_type, int64_t ldx, int T, const uint8_t *codes, const uint16_t *scales, int O, int K,
                   int group, const float *scale, const float *shift, int act, void *y, int y_type, int64_t ldy,
                   const float *add, cudaStream_t s) {
    Args a{};
    a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy; a.codes = codes; a.scales = scales; a.scale = scale; a.shift = shift;
    a.add = add; a.T = T; a.O = O; a.K = K; a.nb = (K + 127) / 128; a.groups = (K + group - 1) / group; a.group = group;
    a.by_blocks = Div(group >= 128 ? group / 128 : 1);
    a.x_bf16 = x_type == MINW_BF16; a.y_bf16 = y_type == MINW_BF16; a.act = act;
    a.parts = a.x_bf16 ? 1 : 3;
    const int most = 32 / a.parts;                                   // vectors of a pass: 32 columns
    a.tokens = T < most ? T : most;
    const int passes = (T + a.tokens - 1) / a.tokens, cols = a.tokens * a.parts, NT = (cols + 7) / 8;
    if (passes > 65535) return MINW_EUNSUPPORTED;
    const int units = (a.nb + 1) / 2, sms = num_sms() > 0 ? num_sms() : 152;
    // wr warps along the rows (16 each) and wk along K make a CTA, `split` CTAs a cluster, which splits K too: the
    // choice with the least estimated clocks.  An SM holds two CTAs of up to 100 KB of shared memory: the rings, and x
    // and scales of as many units (whole rounds of the warps) as fit.  Measured on one to 48 columns (T = 1: 1024 x
    // 1024 to 16384 x 16384): fourteen warps of an SM take 18 / (1 + 0.07 columns) bytes of codes a clock, fewer
    // warps their share of that; a wave of CTAs has a fixed part, so have a cluster and each further filling of x.
    float best = 1e30f;
    // with the share of the SMs' places that clusters of this size can take (cudaOccupancyMaxActiveClusters)
    static const struct { int n; float places; } splits[] = {{1, 1.0f}, {2, 1.0f}, {3, 0.957f}, {4, 0.974f}, {6, 0.908f}, {8, 0.948f}};
    const float x_rate = a.tokens * 256 * (a.x_bf16 ? 0.03f : 0.14f), cap = 18.0f / (1.0f + 0.07f * cols);
    int tiles = 0;
    for (int wr = 1; wr <= WARPS; ++wr) {
        const int wk = WARPS / wr, warps = wr * wk, rows = (O + 16 * wr - 1) / (16 * wr);
        const int room = 100 * 1024 - warps * ring_of(NT) * UNIT_BYTES - cols * 64 - 512 - wr * 16 * 32;
        const int fit = room / (cols * 512 + wr * 32 * (group >= 256 ? 1 : 256 / group));
        const float one = cap * (warps / 14.0f), two = cap * (warps >= 7 ? 1.0f : warps / 7.0f);
        for (const auto &sp : splits) {
            const int split = sp.n, upc = (units + split - 1) / split, slots = (int)(2 * sms * sp.places);
            if (upc * (split - 1) >= units) break;                                // a CTA without a unit
            const int xunits = upc <= fit ? upc : fit / wk * wk;
            if (xunits == 0) continue;
            const float bytes = (float)((upc + wk - 1) / wk * wk * wr * UNIT_BYTES);    // the warps' last units are whole
            const float fixed = 1500.0f * ((upc + xunits - 1) / xunits) + (split > 1 ? 1000.0f : 0.0f);
            const float t1 = bytes / one + upc * x_rate + fixed, t2 = 2 * (bytes / two + upc * x_rate) + fixed;
            const int64_t ctas = (int64_t)rows * split * passes, rest = ctas % slots;
            const float t = (float)(ctas / slots) * t2 + (rest > sms ? t2 : rest > 0 ? t1 : 0.0f);
            if (t < best) {
                best = t;
                a.wr = wr;
                a.wk = wk;
                a.split = split;
                a.upc = upc;
                a.xunits = xunits;
                tiles = rows;
            }
        }
    }
    const int ring = a.wr * a.wk * ring_of(NT) * UNIT_BYTES;
    a.xpitch = a.xunits * 256 + 32;
    a.by_row = Div((uint32_t)a.xunits * (a.x_bf16 ? 32 : 64));
    a.scale_pitch = ((group >= 256 ? a.xunits * 256 / group + 2 : a.xunits * (256 / group)) + 7) / 8 * 8;
    a.by_eights = Div((uint32_t)a.scale_pitch / 8);
    a.scale_at = (cols * a.xpitch + 256) * 2;
    a.ring_at = a.scale_at + a.wr * 16 * a.scale_pitch * 2;
    size_t smem = (size_t)a.ring_at + ring;
    const size_t red = (size_t)a.wr * a.wk * 16 * 8 * NT * sizeof(float);
    if (smem < red) smem = red;
    const dim3 grid((unsigned)(tiles * a.split), (unsigned)passes);
    const cudaError_t e = NT == 1 ? launch_group<1>(a, group, grid, smem, s)
                        : NT == 2 ? launch_group<2>(a, group, grid, smem, s)
                        : NT == 3 ? launch_group<3>(a, group, grid, smem, s)
                                  : launch_group<4>(a, group, grid, smem, s);
    return e == cudaSuccess ? launch_status() : launch_failed();
}

}  // namespace w4
}  // namespace minw

using namespace minw;
using namespace minw_host;

extern "C" {

minw_status minw_pack_w4(const void *w, int32_t type, int32_t O, int32_t K, int32_t group, const minw_quant *q,
                         const float *channel_scale, uint8_t *codes, uint16_t *scales, void *stream) {
    if (!w || !codes || !scales || O < 1 || K < 1 || !w4::valid_group(group)) return MINW_EINVAL;
    if ((type != MINW_F32 && type != MINW_BF16) || (q && !valid_quant(q))) return MINW_EINVAL;
    if (!aligned16(codes) || reinterpret_cast<uintptr_t>(scales) % 2 != 0 || !on_floats(channel_scale) ||
        reinterpret_cast<uintptr_t>(w) % (type == MINW_BF16 ? 2 : 4) != 0)
        return MINW_EINVAL;
    if (K > (1 << 28) || group > (1 << 28)) return MINW_EUNSUPPORTED;
    const int Kp = (K + 127) / 128 * 128;
    if ((int64_t)O * ((Kp + group - 1) / group) * 32 / w4::THREADS >= (1ll << 31) - 1) return MINW_EUNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = type == MINW_BF16 ? w4::pack<uint16_t>(w, O, K, Kp, group, q, channel_scale, codes, scales, s)
                                            : w4::pack<float>(w, O, K, Kp, group, q, channel_scale, codes, scales, s);
    return e == cudaSuccess ? launch_status() : launch_failed();
}

minw_status minw_w4_matvec(const void *x, int32_t x_type, int64_t ldx, int32_t T, const uint8_t *codes,
                           const uint16_t *scales, int32_t O, int32_t K, int32_t group, const float *scale,
                           const float *shift, int32_t act, void *y, int32_t y_type, int64_t ldy, void *stream) {
    const minw_status st = w4::check(x, x_type, ldx, T, codes, scales, O, K, group, scale, shift, act, y, y_type, ldy);
    if (st != MINW_OK || T == 0) return st;
    return w4::matvec(x, x_type, ldx, T, codes, scales, O, K, group, scale, shift, act, y, y_type, ldy, nullptr,
                      (cudaStream_t)stream);
}

}  // extern "C"
