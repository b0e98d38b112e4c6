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
// have to be written to first, at four times their packed bytes.
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

namespace cg = cooperative_groups;

namespace minw {
namespace w4 {

constexpr int THREADS = 256, WARPS = THREADS / 32;

// ---------------------------------------------------------------------------
// Packing
// ---------------------------------------------------------------------------

// S lanes per row and group: the group's largest magnitude, its scale, its codes.
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
    void *y;
    int T, O, K, Kp, groups, gb;       // gb: blocks of 128 values per group (groups of 128 and more)
    int x_bf16, y_bf16, act;
    int parts, tokens;                 // columns of a vector (1, or 3 for fp32), vectors of a pass
    int wr;                            // warps side by side along the rows; the others split K
    int split, bpc;                    // CTAs of a cluster (they split K), blocks of 128 values of each
    int xblocks;                       // blocks of x in shared memory at a time
};

__device__ __forceinline__ uint32_t levels(uint32_t word, int p) {
    uint32_t v = ((word >> (4 * p)) & 0x000f000fu) | 0x43004300u;         // 128 + code, twice
    const uint32_t off = 0x43084308u;                                       // 136
    asm("sub.rn.bf16x2 %0, %0, %1;" : "+r"(v) : "r"(off));
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

__device__ __forceinline__ void copy16(uint16_t *dst, const void *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
                 "r"(bytes)
                 : "memory");
}

// Blocks [b0, b0 + n) of the pass's vectors into shared memory, columns of n 128 + 32 values (the 64 bytes
// over put the eight columns of a tile into different banks), zero past K.
__device__ __forceinline__ void stage(const Args &a, uint16_t *xs, int t0, int tokens, int b0, int n) {
    const int pitch = n * 128 + 32, k0 = b0 * 128, valid = min(a.K - k0, n * 128);
    if (a.x_bf16) {
        const uint16_t *x = static_cast<const uint16_t *>(a.x) + (int64_t)t0 * a.ldx + k0;
        const bool wide = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && a.ldx % 8 == 0;
        for (int t = 0; t < tokens; ++t, x += a.ldx) {
            uint16_t *dst = xs + t * pitch;
            for (int k = 8 * threadIdx.x; k < n * 128; k += 8 * THREADS) {
                const int left = valid - k;
                if (wide) {
                    copy16(dst + k, left > 0 ? x + k : x, left >= 8 ? 16 : left > 0 ? 2 * left : 0);
                } else {
                    uint16_t v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = i < left ? x[k + i] : (uint16_t)0;
                    *reinterpret_cast<uint4 *>(dst + k) =
                        make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16,
                                   v[6] | (uint32_t)v[7] << 16);
                }
            }
        }
        asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
    } else {
        constexpr int U = 4;                                         // loads in flight
        const float *x = static_cast<const float *>(a.x) + (int64_t)t0 * a.ldx + k0;
        const bool wide = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && a.ldx % 4 == 0;
        const int per = n * 32, all = tokens * per;                  // fours of a column, of all
        for (int e0 = threadIdx.x; e0 < all; e0 += U * THREADS) {
            float4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = e0 + u * THREADS, t = e / per, k = 4 * (e - t * per), left = valid - k;
                v[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (e >= all) continue;
                const float *src = x + (int64_t)t * a.ldx + k;
                if (wide && left >= 4) {
                    v[u] = *reinterpret_cast<const float4 *>(src);
                } else {
                    if (left > 0) v[u].x = src[0];
                    if (left > 1) v[u].y = src[1];
                    if (left > 2) v[u].z = src[2];
                    if (left > 3) v[u].w = src[3];
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = e0 + u * THREADS, t = e / per, k = 4 * (e - t * per);
                if (e >= all) break;
                uint16_t p[4][3];
                split3(v[u].x, p[0]);
                split3(v[u].y, p[1]);
                split3(v[u].z, p[2]);
                split3(v[u].w, p[3]);
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    *reinterpret_cast<uint2 *>(xs + (3 * t + i) * pitch + k) =
                        make_uint2(p[0][i] | (uint32_t)p[1][i] << 16, p[2][i] | (uint32_t)p[3][i] << 16);
            }
        }
    }
}

constexpr int DEPTH = 4;              // blocks of 128 values that a warp has in flight

// NT: tiles of 8 columns; FL: words of a lane's four that share a scale (1, 2, 4 for groups of 32, 64, 128 and more).
template <int NT, int FL>
__global__ void __launch_bounds__(THREADS, 2) matvec_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    extern __shared__ __align__(16) uint8_t smem[];
    uint16_t *xs = reinterpret_cast<uint16_t *>(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int wr = warp % a.wr, wk = warp / a.wr, nk = WARPS / a.wr;
    const int rank = blockIdx.x % a.split, tile = blockIdx.x / a.split;
    const int t0 = blockIdx.y * a.tokens, tokens = min(a.tokens, a.T - t0), cols = tokens * a.parts;
    const int row = (tile * a.wr + wr) * 16 + g;
    const int r0 = min(row, a.O - 1), r1 = min(row + 8, a.O - 1);       // rows past the last repeat it and are not stored
    const uint4 *w0 = reinterpret_cast<const uint4 *>(a.codes + (int64_t)r0 * (a.Kp / 2)) + t;
    const uint4 *w1 = reinterpret_cast<const uint4 *>(a.codes + (int64_t)r1 * (a.Kp / 2)) + t;
    const uint16_t *s0 = a.scales + (int64_t)r0 * a.groups, *s1 = a.scales + (int64_t)r1 * a.groups;
    const int first = rank * a.bpc, last = min(a.Kp / 128, first + a.bpc);
    float tot[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) tot[n][i] = 0.0f;

    // codes and scales of the warp's next DEPTH blocks
    uint4 u0[DEPTH], u1[DEPTH];
    uint32_t f0[DEPTH], f1[DEPTH];                                     // lane t: the scale of word t
    auto fetch = [&](int d, int kb) {
        if (kb >= last) return;
        u0[d] = __ldcs(w0 + kb * 4);
        u1[d] = __ldcs(w1 + kb * 4);
        const int sg = FL == 4 ? (a.gb == 1 ? kb : kb / a.gb) : kb * (4 / FL) + t / FL;
        f0[d] = sg < a.groups ? s0[sg] : 0u;                           // a group past the last holds padding only
        f1[d] = sg < a.groups ? s1[sg] : 0u;
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(d, first + wk + d * nk);

    for (int c0 = first; c0 < last; c0 += a.xblocks) {
        const int nb = min(a.xblocks, last - c0), pitch = nb * 128 + 32;
        __syncthreads();
        stage(a, xs, t0, tokens, c0, nb);
        __syncthreads();
        for (int k0 = c0 + wk; k0 < c0 + nb; k0 += DEPTH * nk) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int kb = k0 + d * nk;
                if (kb >= c0 + nb) break;
                const uint32_t q0[4] = {u0[d].x, u0[d].y, u0[d].z, u0[d].w}, q1[4] = {u1[d].x, u1[d].y, u1[d].z, u1[d].w};
                float h0[4 / FL], h1[4 / FL];
#pragma unroll
                for (int s = 0; s < 4 / FL; ++s) {
                    h0[s] = __uint_as_float((FL == 4 ? f0[d] : __shfl_sync(0xffffffffu, f0[d], s * FL, 4)) << 16);
                    h1[s] = __uint_as_float((FL == 4 ? f1[d] : __shfl_sync(0xffffffffu, f1[d], s * FL, 4)) << 16);
                }
                fetch(d, kb + DEPTH * nk);
                float acc[NT][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j % FL == 0) {
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
                    }
                    uint32_t a0[4], a1[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        a0[p] = levels(q0[j], p);
                        a1[p] = levels(q1[j], p);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        uint4 b = make_uint4(0, 0, 0, 0);
                        if (n * 8 + g < cols)
                            b = *reinterpret_cast<const uint4 *>(xs + (n * 8 + g) * pitch + (kb - c0) * 128 + 32 * j + 8 * t);
                        mma(acc[n], a0[0], a1[0], a0[1], a1[1], b.x, b.y);
                        mma(acc[n], a0[2], a1[2], a0[3], a1[3], b.z, b.w);
                    }
                    if (j % FL == FL - 1) {
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            tot[n][0] = fmaf(h0[j / FL], acc[n][0], tot[n][0]);
                            tot[n][1] = fmaf(h0[j / FL], acc[n][1], tot[n][1]);
                            tot[n][2] = fmaf(h1[j / FL], acc[n][2], tot[n][2]);
                            tot[n][3] = fmaf(h1[j / FL], acc[n][3], tot[n][3]);
                        }
                    }
                }
            }
        }
    }

    // the warps' sums [warp][16 rows][8 NT columns], then the cluster's, in a fixed order
    constexpr int CW = 8 * NT;
    float *red = reinterpret_cast<float *>(smem);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float *d = red + (warp * 16 + g) * CW + n * 8 + 2 * t;
        d[0] = tot[n][0];
        d[1] = tot[n][1];
        d[8 * CW] = tot[n][2];
        d[8 * CW + 1] = tot[n][3];
    }
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    const int rows = a.wr * 16, each = (rows + a.split - 1) / a.split, rr0 = rank * each, rr1 = min(rows, rr0 + each);
    for (int e = threadIdx.x; e < (rr1 - rr0) * tokens; e += THREADS) {
        const int r = rr0 + e / tokens, tk = e % tokens, o = tile * rows + r;
        if (o >= a.O) continue;
        float sum = 0.0f;
        for (int i = a.parts - 1; i >= 0; --i)                        // the smallest part first
            for (int c = 0; c < a.split; ++c) {
                const float *src = cluster.map_shared_rank(red, c);
                for (int k = 0; k < nk; ++k)
                    sum += src[((k * a.wr + r / 16) * 16 + r % 16) * CW + tk * a.parts + i];
            }
        float z = fmaf(sum, a.scale ? a.scale[o] : 1.0f, a.shift ? a.shift[o] : 0.0f);
        with_act(a.act, [&](auto act) { z = act_value<act.value>(z); });
        const int64_t at = (int64_t)(t0 + tk) * a.ldy + o;
        if (a.y_bf16) static_cast<uint16_t *>(a.y)[at] = __bfloat16_as_ushort(__float2bfloat16_rn(z));
        else static_cast<float *>(a.y)[at] = z;
    }
    cluster.sync();                                                    // no CTA leaves while its sums are read
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
    cfg.blockDim = dim3(THREADS);
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

}  // namespace w4
}  // namespace minw

using namespace minw;
using namespace minw_host;

extern "C" {

minw_status minw_pack_w4(const void *w, int32_t type, int32_t O, int32_t K, int32_t group, const minw_quant *q,
                         const float *channel_scale, uint8_t *codes, uint16_t *scales, void *stream) {
    if (!w || !codes || !scales || O < 1 || K < 1 || !w4::valid_group(group)) return MINW_EINVAL;
    if ((type != MINW_F32 && type != MINW_BF16) || (q && !valid_quant(q))) return MINW_EINVAL;
    if (!aligned16(codes) || reinterpret_cast<uintptr_t>(scales) % 2 != 0 ||
        reinterpret_cast<uintptr_t>(w) % (type == MINW_BF16 ? 2 : 4) != 0)
        return MINW_EINVAL;
    if (K > (1 << 28) || group > (1 << 28)) return MINW_EUNSUPPORTED;
    const int Kp = (K + 127) / 128 * 128;
    if ((int64_t)O * ((Kp + group - 1) / group) * 32 / w4::THREADS >= (1ll << 31) - 1) return MINW_EUNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = type == MINW_BF16 ? w4::pack<uint16_t>(w, O, K, Kp, group, q, channel_scale, codes, scales, s)
                                            : w4::pack<float>(w, O, K, Kp, group, q, channel_scale, codes, scales, s);
    return e == cudaSuccess ? launch_status() : MINW_ECUDA;
}

minw_status minw_w4_matvec(const void *x, int32_t x_type, int64_t ldx, int32_t T, const uint8_t *codes,
                           const uint16_t *scales, int32_t O, int32_t K, int32_t group, const float *scale,
                           const float *shift, int32_t act, void *y, int32_t y_type, int64_t ldy, void *stream) {
    if (!codes || !scales || (T != 0 && (!x || !y)) || T < 0 || O < 1 || K < 1 || ldx < K || ldy < O) return MINW_EINVAL;
    if (!w4::valid_group(group) || act < MINW_ACT_NONE || act > MINW_ACT_SILU) return MINW_EINVAL;
    if ((x_type != MINW_F32 && x_type != MINW_BF16) || (y_type != MINW_F32 && y_type != MINW_BF16)) return MINW_EINVAL;
    if (!aligned16(codes) || reinterpret_cast<uintptr_t>(scales) % 2 != 0 ||
        reinterpret_cast<uintptr_t>(x) % (x_type == MINW_BF16 ? 2 : 4) != 0 ||
        reinterpret_cast<uintptr_t>(y) % (y_type == MINW_BF16 ? 2 : 4) != 0)
        return MINW_EINVAL;
    if (K > (1 << 28) || group > (1 << 28) || O > (1 << 28)) return MINW_EUNSUPPORTED;
    if (T == 0) return MINW_OK;
    w4::Args a{};
    a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy; a.codes = codes; a.scales = scales; a.scale = scale; a.shift = shift;
    a.T = T; a.O = O; a.K = K; a.Kp = (K + 127) / 128 * 128; a.groups = (K + group - 1) / group;
    a.gb = group >= 128 ? group / 128 : 1;
    a.x_bf16 = x_type == MINW_BF16; a.y_bf16 = y_type == MINW_BF16; a.act = act;
    a.parts = a.x_bf16 ? 1 : 3;
    const int most = 32 / a.parts;                                   // vectors of a pass: 32 columns
    a.tokens = T < most ? T : most;
    const int passes = (T + a.tokens - 1) / a.tokens, cols = a.tokens * a.parts, NT = (cols + 7) / 8;
    if (passes > 65535) return MINW_EUNSUPPORTED;
    const int nb = a.Kp / 128, sms = num_sms() > 0 ? num_sms() : 152;
    // Rows of a CTA (16 for each of wr warps side by side; the other warps split K) and CTAs of a cluster (which split K
    // too): the pair with the least estimated time, waves of two CTAs per SM times a CTA's clocks -- its share of the
    // memory rate for the codes, of L2's for x (fp32 values are split into parts as well), and a fixed part.
    double best = 1e30;
    for (int wr = 1; wr <= w4::WARPS; wr *= 2)
        for (int split = 1; split <= 8; split *= 2) {
            const int64_t tiles = (O + 16 * wr - 1) / (16 * wr);
            const int bpc = (nb + split - 1) / split;
            if (split > 1 && bpc * split - nb >= bpc) continue;                   // a CTA without a block
            const int round = w4::WARPS / wr * w4::DEPTH;                         // x in shared memory: a round at least
            if ((bpc < round ? bpc : round) * cols > 400) continue;               // (100 KB)
            const int steps = (bpc * wr + w4::WARPS - 1) / w4::WARPS * w4::WARPS / wr;     // blocks, the warps' last ones whole
            const double clocks = steps * (wr * 1024 / 11.0) + bpc * a.tokens * 128 * (a.x_bf16 ? 0.06 : 0.28) + 2500;
            const double t = (double)((tiles * split * passes + 2 * sms - 1) / (2 * sms)) * clocks;
            if (t < best) {
                best = t;
                a.wr = wr;
                a.split = split;
                a.bpc = bpc;
            }
        }
    const int tiles = (O + 16 * a.wr - 1) / (16 * a.wr), unit = w4::WARPS / a.wr * w4::DEPTH;
    int xb = 400 / cols;                                             // at most 100 KB of x at a time, whole rounds of the warps
    xb = xb / unit * unit > 0 ? xb / unit * unit : unit;
    a.xblocks = a.bpc < xb ? a.bpc : xb;
    size_t smem = (size_t)cols * (a.xblocks * 128 + 32) * 2;
    const size_t red = (size_t)w4::WARPS * 16 * 8 * NT * sizeof(float);
    if (smem < red) smem = red;
    const dim3 grid((unsigned)(tiles * a.split), (unsigned)passes);
    cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = NT == 1 ? w4::launch_group<1>(a, group, grid, smem, s)
                        : NT == 2 ? w4::launch_group<2>(a, group, grid, smem, s)
                        : NT == 3 ? w4::launch_group<3>(a, group, grid, smem, s)
                                  : w4::launch_group<4>(a, group, grid, smem, s);
    return e == cudaSuccess ? launch_status() : MINW_ECUDA;
}

}  // extern "C"
