// values.cuh -- what the kernels of a head share: vectors of fp32 or bf16 values
// as they lie in memory, fp32 pairs, activations, the end of a cluster, division
// by numbers the host knows.
#pragma once

#include <cuda_bf16.h>

#include <type_traits>

#include "common.cuh"

namespace minw {

// Two fp32 values in a register pair: one instruction for both.
struct Pair {
    uint64_t v;
};
__device__ __forceinline__ Pair pair(float lo, float hi) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ float2 halves(Pair p) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p.v));
    return f;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// V consecutive values of type T (float, or uint16_t holding bf16 bits), one load or store of up to 16 bytes each.
// The address is a multiple of the load's size.
template <typename T, int V>
struct Vec {
    static constexpr int BYTES = V * (int)sizeof(T);
    static constexpr int WORDS = BYTES < 4 ? 1 : BYTES / 4;
    uint32_t w[WORDS];

    __device__ __forceinline__ void load(const T *p) {
        if constexpr (BYTES == 2) {
            w[0] = *reinterpret_cast<const uint16_t *>(p);
        } else if constexpr (BYTES == 4) {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        } else if constexpr (BYTES == 8) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            w[0] = v.x; w[1] = v.y;
        } else {
#pragma unroll
            for (int k = 0; k < WORDS / 4; ++k) {
                const uint4 v = reinterpret_cast<const uint4 *>(p)[k];
                w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
            }
        }
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (BYTES == 2) {
            *reinterpret_cast<uint16_t *>(p) = (uint16_t)w[0];
        } else if constexpr (BYTES == 4) {
            *reinterpret_cast<uint32_t *>(p) = w[0];
        } else if constexpr (BYTES == 8) {
            *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int k = 0; k < WORDS / 4; ++k)
                reinterpret_cast<uint4 *>(p)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float((i & 1) ? (w[i >> 1] & 0xffff0000u) : (w[i >> 1] << 16));
    }
    // values 2 k and 2 k + 1 (0 past a single one)
    __device__ __forceinline__ Pair get2(int k) const { return pair(get(2 * k), V > 1 ? get(2 * k + 1) : 0.0f); }
    // all V values at once: bf16 rounds to nearest even, two to a conversion
    __device__ __forceinline__ void set(const float *v) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = __float_as_uint(v[i]);
        } else if constexpr (V == 1) {
            w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
        } else {
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[i], v[i + 1]);
                w[i >> 1] = *reinterpret_cast<const uint32_t *>(&b);
            }
        }
    }
};

// BYTES (8 or 16) from global to shared memory, asynchronously.
template <int BYTES>
__device__ __forceinline__ void copy_async(void *dst, const void *src) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(d), "l"(src) : "memory");
}

// The larger and the smaller of two values; a NaN among them stays one (fmaxf and fminf drop it).
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 1 / (1 + e^-z): tends to 0 and 1 at both ends (e^-z = infinity gives 0).  Two approximate instructions, each within
// 2 ulp; the argument's rounding adds |z| 2^-24.
__device__ __forceinline__ float sigmoidf_(float z) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return r;
}

// y = act(z); a NaN stays one.
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == MINW_ACT_HARDTANH) return min_nan(max_nan(z, -1.0f), 1.0f);
    if constexpr (ACT == MINW_ACT_RELU) return max_nan(z, 0.0f);
    if constexpr (ACT == MINW_ACT_SILU) return z * sigmoidf_(z);
    return z;
}

// dy act'(z).  HardTanh passes the gradient on |z| <= 1 (Eq. activation's mask), ReLU on z > 0.
template <int ACT>
__device__ __forceinline__ float act_grad(float z, float dy) {
    if constexpr (ACT == MINW_ACT_HARDTANH) return fabsf(z) <= 1.0f ? dy : 0.0f;
    if constexpr (ACT == MINW_ACT_RELU) return z > 0.0f ? dy : 0.0f;
    if constexpr (ACT == MINW_ACT_SILU) {
        const float s = sigmoidf_(z);
        return dy * (s * fmaf(z, 1.0f - s, 1.0f));
    }
    return dy;
}

template <int ACT>
__device__ __forceinline__ Pair act_grad2(Pair z, Pair dy) {
    if constexpr (ACT == MINW_ACT_NONE) return dy;
    const float2 zf = halves(z), df = halves(dy);
    if constexpr (ACT == MINW_ACT_SILU) {
        const Pair s = pair(sigmoidf_(zf.x), sigmoidf_(zf.y)), one = pair(1.0f, 1.0f);
        return mul2(dy, mul2(s, fma2(z, fma2(s, pair(-1.0f, -1.0f), one), one)));
    }
    return pair(act_grad<ACT>(zf.x, df.x), act_grad<ACT>(zf.y, df.y));
}

// The end of a cluster: no block leaves while others read its shared memory.  Arriving needs no memory ordering, the
// values read have been used by then.
__device__ __forceinline__ void cluster_done_reading() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_leave() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }

// n / d for 0 <= n < 2^31 with the divisor (1 to 2^31) known on the host: a product's upper half and a shift.
struct Div {
    uint32_t d = 1, m = 1, s = 0;
    Div() = default;
    explicit Div(uint32_t by) : d(by) {
        while ((1ull << s) < by) ++s;
        m = (uint32_t)(((1ull << 32) * ((1ull << s) - by)) / by + 1);
    }
    __device__ __forceinline__ int div(int n) const { return (int)((__umulhi(m, (uint32_t)n) + (uint32_t)n) >> s); }
};

// f(std::integral_constant<int, act>): the choice once around a loop, not at each value.
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    if (act == MINW_ACT_HARDTANH) f(std::integral_constant<int, MINW_ACT_HARDTANH>{});
    else if (act == MINW_ACT_RELU) f(std::integral_constant<int, MINW_ACT_RELU>{});
    else if (act == MINW_ACT_SILU) f(std::integral_constant<int, MINW_ACT_SILU>{});
    else f(std::integral_constant<int, MINW_ACT_NONE>{});
}

}  // namespace minw

namespace minw_host {

// Whether every fp32 vector (null: not given) lies on its elements' boundary.
template <typename... T>
inline bool on_floats(const T *...p) {
    return ((reinterpret_cast<uintptr_t>(p) | ...) & 3) == 0;
}

// The status of a launch that the runtime refused, whose error would else be the next call's.
inline minw_status launch_failed() {
    cudaGetLastError();
    return MINW_ECUDA;
}

}  // namespace minw_host
