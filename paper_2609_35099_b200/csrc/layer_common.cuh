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

// V consecutive elements as float32, read or written in one access (V = 1, or 4, 8 or 16 bytes that start on a multiple of
// their size).
template <class T, int V> struct Pack;
template <> struct Pack<float, 1> {
    static __device__ __forceinline__ void load(float (&v)[1], const float* p) { v[0] = __ldg(p); }
    static __device__ __forceinline__ void store(float* p, const float (&v)[1]) { *p = v[0]; }
};
template <> struct Pack<float, 4> {
    static __device__ __forceinline__ void load(float (&v)[4], const float* p) {
        const float4 q = __ldg(reinterpret_cast<const float4*>(p));
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    }
    static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <> struct Pack<bf16, 1> {
    static __device__ __forceinline__ void load(float (&v)[1], const bf16* p) { v[0] = to_float(*p); }
    static __device__ __forceinline__ void store(bf16* p, const float (&v)[1]) { *p = from_float<bf16>(v[0]); }
};
template <> struct Pack<bf16, 2> {
    static __device__ __forceinline__ void load(float (&v)[2], const bf16* p) {
        const uint32_t q = __ldg(reinterpret_cast<const uint32_t*>(p));
        v[0] = low_float(q); v[1] = high_float(q);
    }
    static __device__ __forceinline__ void store(bf16* p, const float (&v)[2]) {
        *reinterpret_cast<uint32_t*>(p) = pack_bf16(v[0], v[1]);
    }
};
template <> struct Pack<bf16, 4> {
    static __device__ __forceinline__ void load(float (&v)[4], const bf16* p) {
        const uint2 q = __ldg(reinterpret_cast<const uint2*>(p));
        v[0] = low_float(q.x); v[1] = high_float(q.x); v[2] = low_float(q.y); v[3] = high_float(q.y);
    }
    static __device__ __forceinline__ void store(bf16* p, const float (&v)[4]) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    }
};
template <> struct Pack<bf16, 8> {
    static __device__ __forceinline__ void load(float (&v)[8], const bf16* p) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
        v[0] = low_float(q.x); v[1] = high_float(q.x); v[2] = low_float(q.y); v[3] = high_float(q.y);
        v[4] = low_float(q.z); v[5] = high_float(q.z); v[6] = low_float(q.w); v[7] = high_float(q.w);
    }
    static __device__ __forceinline__ void store(bf16* p, const float (&v)[8]) {
        *reinterpret_cast<uint4*>(p) =
            make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
};

// 1 / (1 + exp(-z)).  The fast exponential and division are within a few float32 roundings where the result is not tiny;
// exp(-z) = infinity gives 0.
__device__ __forceinline__ float logistic(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

__device__ __forceinline__ float normal_cdf(float z) { return 0.5f * (1.f + erff(0.70710678f * z)); }

template <int ACT> __device__ __forceinline__ float activation(float z) {
    if constexpr (ACT == E3J_ACT_SILU) return z * logistic(z);
    else if constexpr (ACT == E3J_ACT_TANH) return tanhf(z);
    else if constexpr (ACT == E3J_ACT_GELU) return z * normal_cdf(z);
    else return z;
}
template <int ACT> __device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == E3J_ACT_SILU) {
        const float s = logistic(z);
        return s * fmaf(z, 1.f - s, 1.f);
    } else if constexpr (ACT == E3J_ACT_TANH) {
        const float t = tanhf(z);
        return fmaf(-t, t, 1.f);
    } else if constexpr (ACT == E3J_ACT_GELU) {
        return fmaf(z, 0.39894228f * __expf(-0.5f * z * z), normal_cdf(z));
    } else {
        return 1.f;
    }
}
// The same with the activation as a run-time value: one uniform branch for all elements of v.
template <int N> __device__ __forceinline__ void activate(float (&v)[N], int act) {
    if (act == E3J_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activation<E3J_ACT_SILU>(v[i]);
    } else if (act == E3J_ACT_TANH) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activation<E3J_ACT_TANH>(v[i]);
    } else if (act == E3J_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activation<E3J_ACT_GELU>(v[i]);
    }
}
// g[i] *= slope(z[i])
template <int N> __device__ __forceinline__ void times_slope(float (&g)[N], const float (&z)[N], int act) {
    if (act == E3J_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] *= slope<E3J_ACT_SILU>(z[i]);
    } else if (act == E3J_ACT_TANH) {
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] *= slope<E3J_ACT_TANH>(z[i]);
    } else if (act == E3J_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] *= slope<E3J_ACT_GELU>(z[i]);
    }
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
