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
// memory (Raw), and as pairs of float32 (one element: the first of a pair, and 0).  (store_four: four elements, to a multiple of their size.)
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
    // ones in the bits of the elements that f names; masking with them; storing those elements alone
    template <class F> static __device__ __forceinline__ Raw ones(F f) {
        const float one = __uint_as_float(~0u);
        return make_float4(f(0) ? one : 0.f, f(1) ? one : 0.f, f(2) ? one : 0.f, f(3) ? one : 0.f);
    }
    static __device__ __forceinline__ float masked(float v, float m) { return __uint_as_float(__float_as_uint(v) & __float_as_uint(m)); }
    template <int N, class M> static __device__ __forceinline__ void mask(Raw (&r)[N], const M& m) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            r[i] = make_float4(masked(r[i].x, m.r[i].x), masked(r[i].y, m.r[i].y), masked(r[i].z, m.r[i].z), masked(r[i].w, m.r[i].w));
    }
    static __device__ __forceinline__ void store_inside(float* p, const Raw& r, const Raw& m) {
        if (__float_as_uint(m.x)) p[0] = r.x;
        if (__float_as_uint(m.y)) p[1] = r.y;
        if (__float_as_uint(m.z)) p[2] = r.z;
        if (__float_as_uint(m.w)) p[3] = r.w;
    }
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
    template <class F> static __device__ __forceinline__ Raw ones(F f) {
        Raw m;
#pragma unroll
        for (int i = 0; i < 4; ++i) m.w[i] = (f(2 * i) ? 0xffffu : 0u) | (f(2 * i + 1) ? 0xffff0000u : 0u);
        return m;
    }
    template <int N, class M> static __device__ __forceinline__ void mask(Raw (&r)[N], const M& m) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) r[i].w[k] &= m.r[i].w[k];
    }
    static __device__ __forceinline__ void store_inside(bf16* p, const Raw& r, const Raw& m) {
        uint16_t* const h = reinterpret_cast<uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // (a pair at a time where both are inside)
            if (m.w[i] == ~0u) *reinterpret_cast<uint32_t*>(h + 2 * i) = r.w[i];
            if (m.w[i] == 0xffffu) h[2 * i] = (uint16_t)r.w[i];
            if (m.w[i] == 0xffff0000u) h[2 * i + 1] = (uint16_t)(r.w[i] >> 16);
        }
    }
};
__device__ __forceinline__ void store_four(float* p, const float2 (&v)[2]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
}
__device__ __forceinline__ void store_four(bf16* p, const float2 (&v)[2]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y));
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
// Activations and their slopes, on pairs: what can be packed is one instruction for two elements.
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
// 1 / (1 + exp(-z)); exp(-z) = infinity gives 0
__device__ __forceinline__ float2 logistic(float2 z) {
    const float2 x = __fmul2_rn(z, both(-kLog2e));
    const float2 d = __fadd2_rn(make_float2(fast_exp2(x.x), fast_exp2(x.y)), both(1.f));
    return make_float2(fast_reciprocal(d.x), fast_reciprocal(d.y));
}
// Normal distribution: Phi(-|z|), and e = exp(-z^2 / 2), for bfloat16 results.  The rational approximation of Hastings for erf (Abramowitz
// and Stegun 7.1.26), 1 - (a1 t + .. + a5 t^5) exp(-x^2) with t = 1 / (1 + p x) and x = |z| / sqrt 2, which is within 1.5e-7: far
// below half a step of bfloat16, but 2.5 half steps of float32 at 1, and more of what is smaller.
__device__ __forceinline__ float2 normal_exp(float2 z) {
    const float2 x = __fmul2_rn(__fmul2_rn(z, z), both(-0.5f * kLog2e));
    return make_float2(fast_exp2(x.x), fast_exp2(x.y));
}
__device__ __forceinline__ float2 normal_tail(float2 z, float2& e) {
    e = normal_exp(z);
    const float2 t = make_float2(fast_reciprocal(fmaf(0.23164189f, fabsf(z.x), 1.f)), fast_reciprocal(fmaf(0.23164189f, fabsf(z.y), 1.f)));
    float2 poly = __ffma2_rn(both(0.5f * 1.061405429f), t, both(0.5f * -1.453152027f));
    poly = __ffma2_rn(poly, t, both(0.5f * 1.421413741f));
    poly = __ffma2_rn(poly, t, both(0.5f * -0.284496736f));
    poly = __ffma2_rn(poly, t, both(0.5f * 0.254829592f));
    return __fmul2_rn(__fmul2_rn(poly, t), e);
}
// The same for float32 results, by two least-maximum fits of our own in float64 (weighted least squares, the weights moved to where
// the error is largest): near 0, |z| < kNearZero, Phi(z) - 1/2 = z Q(z^2) (relative error 3e-9), beyond it
// Phi(-|z|) = e t P(t), t = 1 / (1 + 0.4 |z|) (6e-8 of the tail).  Both are evaluated, the caller takes one.  2-norm of GELU's error over
// normal values 3.5e-8 (z (1 + erf(z / sqrt 2)) / 2 in float32: 3.8e-8; by Hastings 9e-8, 22e-8 for values a tenth of that).
constexpr float kNearZero = 1.5f;
__device__ __forceinline__ void normal_parts(float2 z, float2& e, float2& middle, float2& tail) {
    e = normal_exp(z);
    const float2 s = __fmul2_rn(z, z);
    float2 q = __ffma2_rn(both(4.1385521853953833e-07f), s, both(-8.733937647775747e-06f));
    q = __ffma2_rn(q, s, both(1.1439632362453267e-04f));
    q = __ffma2_rn(q, s, both(-1.1865355772897601e-03f));
    q = __ffma2_rn(q, s, both(9.973266161978245e-03f));
    q = __ffma2_rn(q, s, both(-6.649033725261688e-02f));
    middle = __ffma2_rn(q, s, both(0.3989422917366028f));   // Q: (Phi(z) - 1/2) / z
    const float2 t = make_float2(fast_reciprocal(fmaf(0.4f, fabsf(z.x), 1.f)), fast_reciprocal(fmaf(0.4f, fabsf(z.y), 1.f)));
    float2 p = __ffma2_rn(both(0.06783036142587662f), t, both(-0.18598994612693787f));
    p = __ffma2_rn(p, t, both(0.1051749661564827f));
    p = __ffma2_rn(p, t, both(0.05552689731121063f));
    p = __ffma2_rn(p, t, both(0.13903166353702545f));
    p = __ffma2_rn(p, t, both(0.15909291803836823f));
    p = __ffma2_rn(p, t, both(0.1595963090658188f));
    tail = __fmul2_rn(__fmul2_rn(p, t), e);
}
// |z|, but finite: beyond 20 Phi(-|z|) is 0 in float32, and infinity times 0 is not what GELU leaves of infinity
__device__ __forceinline__ float size(float z) { return fminf(fabsf(z), 20.f); }
// GELU and its slope (of one element) from those parts: near 0 z / 2 + z (z Q), elsewhere as above; Phi(z) + z phi(z).
__device__ __forceinline__ float2 gelu_of(float2 z, float2 middle, float2 tail) {
    const float2 near = __ffma2_rn(z, __fmul2_rn(z, middle), __fmul2_rn(z, both(0.5f)));
    return make_float2(fabsf(z.x) < kNearZero ? near.x : fmaf(-size(z.x), tail.x, fmaxf(z.x, 0.f)),
                       fabsf(z.y) < kNearZero ? near.y : fmaf(-size(z.y), tail.y, fmaxf(z.y, 0.f)));
}
__device__ __forceinline__ float gelu_slope_of(float z, float e, float middle, float tail) {
    const float density = e * 0.39894228f;
    const bool near = fabsf(z) < kNearZero;
    return fmaf(z, near ? middle + density : density, near ? 0.5f : z > 0.f ? 1.f - tail : tail);
}
// FINE: for float32 results (GELU alone has two forms)
template <int ACT, bool FINE> __device__ __forceinline__ float2 activation(float2 z) {
    if constexpr (ACT == E3J_ACT_SILU) return __fmul2_rn(z, logistic(z));
    else if constexpr (ACT == E3J_ACT_TANH) return make_float2(tanhf(z.x), tanhf(z.y));
    else if constexpr (ACT == E3J_ACT_GELU && FINE) {
        float2 e, middle, tail;
        normal_parts(z, e, middle, tail);
        return gelu_of(z, middle, tail);
    } else if constexpr (ACT == E3J_ACT_GELU) {   // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
        float2 e;
        const float2 tail = normal_tail(z, e);
        return make_float2(fmaf(-size(z.x), tail.x, fmaxf(z.x, 0.f)), fmaf(-size(z.y), tail.y, fmaxf(z.y, 0.f)));
    } else return z;
}
template <int ACT, bool FINE> __device__ __forceinline__ float2 slope(float2 z) {
    if constexpr (ACT == E3J_ACT_SILU) {   // s (1 + z (1 - s))
        const float2 s = logistic(z);
        return __fmul2_rn(s, __ffma2_rn(z, __ffma2_rn(s, both(-1.f), both(1.f)), both(1.f)));
    } else if constexpr (ACT == E3J_ACT_TANH) {
        const float2 t = make_float2(tanhf(z.x), tanhf(z.y));
        return __ffma2_rn(__fmul2_rn(t, both(-1.f)), t, both(1.f));
    } else if constexpr (ACT == E3J_ACT_GELU && FINE) {
        float2 e, middle, tail;
        normal_parts(z, e, middle, tail);
        return make_float2(gelu_slope_of(z.x, e.x, middle.x, tail.x), gelu_slope_of(z.y, e.y, middle.y, tail.y));
    } else if constexpr (ACT == E3J_ACT_GELU) {   // Phi(z) + z phi(z)
        float2 e;
        const float2 beyond = __ffma2_rn(normal_tail(z, e), both(-1.f), both(0.5f));   // 1/2 - Phi(-|z|)
        const float2 Phi = __fadd2_rn(make_float2(copysignf(beyond.x, z.x), copysignf(beyond.y, z.y)), both(0.5f));
        return __ffma2_rn(z, __fmul2_rn(e, both(0.39894228f)), Phi);
    } else return both(1.f);
}
// (T: the type that the results are rounded to)
template <int ACT, class T, int N> __device__ __forceinline__ void activate_as(float2 (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = activation<ACT, sizeof(T) == 4>(v[i]);
}
// g[i] *= slope(z[i])
template <int ACT, class T, int N> __device__ __forceinline__ void times_slope_as(float2 (&g)[N], const float2 (&z)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = __fmul2_rn(g[i], slope<ACT, sizeof(T) == 4>(z[i]));
}
// The same with the activation as a run-time value: one uniform branch for all elements.
template <class T, int N> __device__ __forceinline__ void activate(float2 (&v)[N], int act) {
    if (act == E3J_ACT_SILU) activate_as<E3J_ACT_SILU, T>(v);
    else if (act == E3J_ACT_TANH) activate_as<E3J_ACT_TANH, T>(v);
    else if (act == E3J_ACT_GELU) activate_as<E3J_ACT_GELU, T>(v);
}
template <class T, int N> __device__ __forceinline__ void times_slope(float2 (&g)[N], const float2 (&z)[N], int act) {
    if (act == E3J_ACT_SILU) times_slope_as<E3J_ACT_SILU, T>(g, z);
    else if (act == E3J_ACT_TANH) times_slope_as<E3J_ACT_TANH, T>(g, z);
    else if (act == E3J_ACT_GELU) times_slope_as<E3J_ACT_GELU, T>(g, z);
}

// launch_dependent with clusters of that many blocks.
template <class... KArgs, class... Args>
inline int launch_cluster(void (*kernel)(KArgs...), int blocks, int cluster, int threads, size_t smem, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3((unsigned)threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
    g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err != cudaSuccess ? err : cudaGetLastError());
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
