// split.cuh -- fp32 values as sums of three bf16 parts for the tensor cores'
// warp-wide products: eight values of a row at a time, paired up along the
// row or across two rows.
#pragma once

#include <cuda_bf16.h>

#include "values.cuh"

namespace minw {

template <typename V>
constexpr int parts_of() { return sizeof(V) == 2 ? 1 : 3; }

// Words on from byte `by` (a multiple of the values' size, below 16) of N + 4 words.
template <int N>
__device__ __forceinline__ void shifted(uint32_t *w, int by) {
#pragma unroll
    for (int k = 0; k < N + 2; ++k) w[k] = by & 8 ? w[k + 2] : w[k];
#pragma unroll
    for (int k = 0; k < N + 1; ++k) w[k] = by & 4 ? w[k + 1] : w[k];
#pragma unroll
    for (int k = 0; k < N; ++k) w[k] = by & 2 ? __funnelshift_r(w[k], w[k + 1], 16) : w[k];
}

// Eight consecutive values as they lie in memory; zeros from `left` on.
template <typename V>
struct Eight {
    static constexpr int WORDS = 2 * (int)sizeof(V);
    uint32_t w[WORDS];

    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) w[k] = 0u;
    }
    __device__ __forceinline__ void cut(int left) {
        if (left >= 8) return;
        if constexpr (sizeof(V) == 4) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k >= left) w[k] = 0u;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = 2 * k >= left ? 0u : 2 * k + 1 >= left ? w[k] & 0xffffu : w[k];
        }
    }
    // ODD: off 16-byte boundaries, the aligned sixteens that hold values of these are read and shifted (value by value: twice
    // the time and more).  On them, a sixteen is read that holds some.
    template <bool ODD>
    __device__ __forceinline__ void load(const V *p, int left) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p), first = ODD ? at & ~(uintptr_t)15 : at,
                        end = at + (left < 8 ? left : 8) * (int)sizeof(V);
        constexpr int N = WORDS + (ODD ? 4 : 0);
        uint32_t u[WORDS + 4];
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            uint4 q = make_uint4(0u, 0u, 0u, 0u);
            if (left > 0 && first + 4 * k < end) q = *reinterpret_cast<const uint4 *>(first + 4 * k);
            u[k] = q.x; u[k + 1] = q.y; u[k + 2] = q.z; u[k + 3] = q.w;
        }
        if constexpr (ODD) shifted<WORDS>(u, (int)(at & 15));
#pragma unroll
        for (int k = 0; k < WORDS; ++k) w[k] = u[k];
        cut(left);
    }
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {          // a in the lower half
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// Two fp32 values as pairs of bf16 parts whose sums they are, each part rounded to nearest: what is left after one is 2^-9 of
// the value at most, after two 2^-18 (parts cut off instead leave up to 2^-7 and 2^-15, and products without the smallest
// are 2^-21 off).  An infinity, a NaN or a value past 3.39e38 makes the second part a NaN.
__device__ __forceinline__ void split2(uint32_t a, uint32_t b, uint32_t *p) {
    float x = __uint_as_float(a), y = __uint_as_float(b);
    p[0] = bf16_pair(x, y);
    x -= __uint_as_float(p[0] << 16);
    y -= __uint_as_float(p[0] & 0xffff0000u);
    p[1] = bf16_pair(x, y);
    p[2] = bf16_pair(x - __uint_as_float(p[1] << 16), y - __uint_as_float(p[1] & 0xffff0000u));
}

// Pairs of neighbours of one row: pair k = values 2k, 2k + 1, in parts.
template <typename V>
__device__ __forceinline__ void along(const Eight<V> &e, uint32_t (*p)[4]) {
    if constexpr (sizeof(V) == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) p[0][k] = e.w[k];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t s[3];
            split2(e.w[2 * k], e.w[2 * k + 1], s);
#pragma unroll
            for (int i = 0; i < 3; ++i) p[i][k] = s[i];
        }
    }
}

// Pairs across two rows: value i of the first and of the second, in parts.
template <typename V>
__device__ __forceinline__ void across(const Eight<V> &a, const Eight<V> &b, int i, uint32_t *p) {
    if constexpr (sizeof(V) == 2) p[0] = __byte_perm(a.w[i >> 1], b.w[i >> 1], (i & 1) ? 0x7632 : 0x5410);
    else split2(a.w[i], b.w[i], p);
}

__device__ __forceinline__ void mma16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

}  // namespace minw
