// What the radial network's hidden layers (linear.cu, layer_norm.cu) share: element types, accesses of several elements,
// activations and their slopes.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "common.cuh"
#include "fast/fast_common.cuh"

namespace e3j {
namespace layer {

using bf16 = __nv_bfloat16;

// Rows [0, real) of a call are real, those behind them padding (n_real null: there are none).
__device__ __forceinline__ int64_t real_rows(int64_t rows, const int32_t* n_real) {
    return n_real ? min(max((int64_t)*n_real, (int64_t)0), rows) : rows;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float v) { return __float2bfloat16_rn(v); }
// two bfloat16 in a register, as they lie in memory
__device__ __forceinline__ float low_float(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high_float(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// V consecutive elements, read or written in one access (16 bytes that start on a multiple of 16, or one element): as they lie in
// memory (Raw), and as pairs of float32 (one element: the first of a pair, and 0).
template <class T, int V> struct Pack;
template <> struct Pack<float, 1> {
    using Raw = float;
    static constexpr int kPairs = 1;
    static __device__ __forceinline__ Raw none() { return 0.f; }
    static __device__ __forceinline__ Raw fetch(const float* p) { return __ldg(p); }
    static __device__ __forceinline__ float2 pair(const Raw& r, int) { return make_float2(r, 0.f); }
    static __device__ __forceinline__ Raw from(const float2 (&v)[1]) { return v[0].x; }
    static __device__ __forceinline__ void store(float* p, const Raw& r) { *p = r; }
};
template <> struct Pack<float, 4> {
    using Raw = float4;
    static constexpr int kPairs = 2;
    static __device__ __forceinline__ Raw none() { return make_float4(0.f, 0.f, 0.f, 0.f); }
    static __device__ __forceinline__ Raw fetch(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
    static __device__ __forceinline__ float2 pair(const Raw& q, int i) { return i ? make_float2(q.z, q.w) : make_float2(q.x, q.y); }
    static __device__ __forceinline__ Raw from(const float2 (&v)[2]) { return make_float4(v[0].x, v[0].y, v[1].x, v[1].y); }
    static __device__ __forceinline__ void store(float* p, const Raw& r) { *reinterpret_cast<float4*>(p) = r; }
};
template <> struct Pack<bf16, 1> {
    using Raw = uint16_t;
    static constexpr int kPairs = 1;
    static __device__ __forceinline__ Raw none() { return 0; }
    static __device__ __forceinline__ Raw fetch(const bf16* p) { return __ldg(reinterpret_cast<const uint16_t*>(p)); }
    static __device__ __forceinline__ float2 pair(const Raw& r, int) { return make_float2(low_float(r), 0.f); }
    static __device__ __forceinline__ Raw from(const float2 (&v)[1]) { return (uint16_t)pack_bf16(v[0].x, 0.f); }
    static __device__ __forceinline__ void store(bf16* p, const Raw& r) { *reinterpret_cast<uint16_t*>(p) = r; }
};
template <> struct Pack<bf16, 8> {
    struct Raw { uint32_t w[4]; };
    static constexpr int kPairs = 4;
    static __device__ __forceinline__ Raw none() { return Raw{{0, 0, 0, 0}}; }
    static __device__ __forceinline__ Raw fetch(const bf16* p) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
        return Raw{{q.x, q.y, q.z, q.w}};
    }
    static __device__ __forceinline__ float2 pair(const Raw& q, int i) { return make_float2(low_float(q.w[i]), high_float(q.w[i])); }
    static __device__ __forceinline__ Raw from(const float2 (&v)[4]) {
        return Raw{{pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y), pack_bf16(v[2].x, v[2].y), pack_bf16(v[3].x, v[3].y)}};
    }
    static __device__ __forceinline__ void store(bf16* p, const Raw& r) {
        *reinterpret_cast<uint4*>(p) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    }
};
// Four elements that start on a multiple of their size.
__device__ __forceinline__ void load_four(float (&v)[4], const float* p) {
    const float4 q = __ldg(reinterpret_cast<const float4*>(p));
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
}
__device__ __forceinline__ void load_four(float (&v)[4], const bf16* p) {
    const uint2 q = __ldg(reinterpret_cast<const uint2*>(p));
    v[0] = low_float(q.x); v[1] = high_float(q.x); v[2] = low_float(q.y); v[3] = high_float(q.y);
}
__device__ __forceinline__ void store_four(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store_four(bf16* p, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
}

// 2^x and 1 / x by the hardware's approximations (within 2 and 1 steps of float32; results below the normal range are 0).
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fast_reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.44269504f;
// 1 / (1 + exp(-z)); exp(-z) = infinity gives 0
__device__ __forceinline__ float logistic(float z) { return fast_reciprocal(1.f + fast_exp2(-kLog2e * z)); }

// Normal distribution: its density phi(z) and distribution function Phi(z) from one exponential.  erf by the rational approximation
// of Hastings (Abramowitz and Stegun 7.1.26), 1 - (a1 t + .. + a5 t^5) exp(-x^2) with t = 1 / (1 + p x), which is within 1.5e-7
// (2.5 half steps of float32); Phi of a negative z is the second term's half and keeps its relative accuracy.  A layer norm of
// 49 157 rows of 385 bfloat16 with GELU is bound by instructions: backward NNN us, with erff MMM.
__device__ __forceinline__ void normal(float z, float& phi, float& Phi) {
    const float x = fabsf(z) * 0.70710678f;
    const float t = fast_reciprocal(fmaf(0.3275911f, x, 1.f));
    const float e = fast_exp2(-kLog2e * x * x);
    float poly = fmaf(1.061405429f, t, -1.453152027f);
    poly = fmaf(poly, t, 1.421413741f);
    poly = fmaf(poly, t, -0.284496736f);
    poly = fmaf(poly, t, 0.254829592f);
    const float tail = 0.5f * poly * t * e;   // Phi(-|z|)
    Phi = z < 0.f ? tail : 1.f - tail;
    phi = 0.39894228f * e;
}

template <int ACT> __device__ __forceinline__ float activation(float z) {
    if constexpr (ACT == E3J_ACT_SILU) return z * logistic(z);
    else if constexpr (ACT == E3J_ACT_TANH) return tanhf(z);
    else if constexpr (ACT == E3J_ACT_GELU) {
        float phi, Phi;
        normal(z, phi, Phi);
        return z * Phi;
    } else return z;
}
template <int ACT> __device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == E3J_ACT_SILU) {
        const float s = logistic(z);
        return s * fmaf(z, 1.f - s, 1.f);
    } else if constexpr (ACT == E3J_ACT_TANH) {
        const float t = tanhf(z);
        return fmaf(-t, t, 1.f);
    } else if constexpr (ACT == E3J_ACT_GELU) {
        float phi, Phi;
        normal(z, phi, Phi);
        return fmaf(z, phi, Phi);
    } else {
        return 1.f;
    }
}
// The same with the activation as a run-time value: one uniform branch for all elements.
template <int ACT, int N> __device__ __forceinline__ void activate_as(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = activation<ACT>(v[i]);
}
template <int ACT, int N> __device__ __forceinline__ void activate_as(float2 (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = make_float2(activation<ACT>(v[i].x), activation<ACT>(v[i].y));
}
template <class F, int N> __device__ __forceinline__ void activate(F (&v)[N], int act) {
    if (act == E3J_ACT_SILU) activate_as<E3J_ACT_SILU>(v);
    else if (act == E3J_ACT_TANH) activate_as<E3J_ACT_TANH>(v);
    else if (act == E3J_ACT_GELU) activate_as<E3J_ACT_GELU>(v);
}
// g[i] *= slope(z[i])
template <int ACT, int N> __device__ __forceinline__ void times_slope_as(float (&g)[N], const float (&z)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] *= slope<ACT>(z[i]);
}
template <int ACT, int N> __device__ __forceinline__ void times_slope_as(float2 (&g)[N], const float2 (&z)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = __fmul2_rn(g[i], make_float2(slope<ACT>(z[i].x), slope<ACT>(z[i].y)));
}
template <class F, int N> __device__ __forceinline__ void times_slope(F (&g)[N], const F (&z)[N], int act) {
    if (act == E3J_ACT_SILU) times_slope_as<E3J_ACT_SILU>(g, z);
    else if (act == E3J_ACT_TANH) times_slope_as<E3J_ACT_TANH>(g, z);
    else if (act == E3J_ACT_GELU) times_slope_as<E3J_ACT_GELU>(g, z);
}

// A parameter's gradient from the blocks' shares of it, added in a fixed order: 32 elements a block, kSumWays
// threads take every kSumWays-th share of an element, their sums are added in order.  Two parameters of n elements
// (second null: one) whose shares lie behind one another, [shares][elements].
constexpr int kSumWays = 16;
template <class T>
__global__ void __launch_bounds__(32 * kSumWays)
sum_shares_kernel(int n_shares, int64_t elements, int64_t n_first, const float* __restrict__ shares, T* __restrict__ first,
                  T* __restrict__ second) {
    __shared__ float part[kSumWays][32];
    const int64_t i = (int64_t)blockIdx.x * 32 + threadIdx.x;
    fast::grid_dependency_wait();
    float sum = 0.f;
    if (i < elements)
        for (int s = threadIdx.y; s < n_shares; s += kSumWays) sum += shares[(int64_t)s * elements + i];
    part[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.y == 0 && i < elements) {
        for (int w = 1; w < kSumWays; ++w) sum += part[w][threadIdx.x];
        T* const to = i < n_first ? first + i : second + (i - n_first);
        if (i < n_first ? first != nullptr : second != nullptr) *to = from_float<T>(sum);
    }
}
template <class T>
inline int sum_shares(int n_shares, int64_t n_first, int64_t n_second, const float* shares, T* first, T* second, cudaStream_t st) {
    const int64_t elements = n_first + n_second;
    return launch_dependent(sum_shares_kernel<T>, dim3((unsigned)((elements + 31) / 32)), dim3(32, kSumWays), 0, st, n_shares,
                            elements, n_first, shares, first, second);
}

}  // namespace layer
}  // namespace e3j
